// Tree-masked verification attention over a latent paged cache (latent.hip writes it): every
// query head of a request reads the same rows of 576 values, all of a row as its key and
// dims 0-511 as its value.  Two launches, and one more before them for large block tables:
//
//   latent_pages    checks the page ids (small tables: the main kernel's workgroups do).
//   latent_main     persistent, one workgroup of four waves per CU.  A unit is up to 128 of a
//                   request's rows (verify slots x heads, which lie one after another), 64
//                   where there is little work; its
//                   tiles are 32 keys each, first the tree's, then the prefix's.  The tiles
//                   of all units are cut into ranges of equal cost, one per workgroup, which
//                   every workgroup finds by itself from the requests' lengths; where that
//                   is faster, a range is a whole unit.
//                   A tile is copied HBM -> LDS once and used twice.  S^T = K Q^T: each wave
//                   has 32 (or 16) rows, its part of Q stays in registers.  The weights go
//                   through LDS.  O^T += V^T P^T: each wave has 128 of the 512 dims for all
//                   rows, so that a fragment of V serves all of them.
//   latent_combine  merges the partial sums of units that several workgroups share.
//
// Softmax statistics and sums are fp32, and so are stored partial sums.  For the product with V
// the weights p are rounded to bfloat16.  A unit of up to 32 rows fills one of the two row tiles that
// its products have anyway: the other takes the same rows' p - bf16(p), summed into the same O, so that
// 2^-16 of p is left, in no more time (a tile 1.02 us for 1.02 with 16 rows, 1.17 for 1.17 with 32,
// nothing of it from HBM; 100 single tokens of 32 heads 42.7 us for 42.1).  Larger units leave
// 2^-8 and divide by the sum of the weights used, so that the output stays a convex
// combination of V rows; the output's own rounding to bfloat16 is as large.  There the rests would be
// products of their own: in units of 64 rows a tile takes 1.45 us instead of 1.17 (64 single tokens of
// 16 heads 92 us for 81, 4 trees 20.6 for 20.0), in units of 128 half as many products again and 16 KB of
// LDS, of which 2 are left.
//
// What bounds it.  A row of 1152 bytes serves 2176 operations per query row, so that up to
// 64 rows are bound by the copies: a tile takes 1.55 us on every CU at once, 6.1 TB/s,
// of 1.0 us of work.  128 rows are bound by the products: 2177 cycles of a CU's
// matrix cores of the 4050 that a tile takes (1.9 us, 2.3 where nothing of it is in a
// cache and the clock is lower).  A wave is alone on its SIMD and issues an instruction in
// four cycles at best: of the 600 of a step those between products run in their shadow,
// the others, its start and its end, cost their own time.  Eight waves with half the rows each
// hide more and read every fragment twice: 755 against 727 us for 16 long requests, 210
// against 192 for 128 trees.  Entering a unit costs 8 us (to 64 rows) to 20 (128: its
// 147 KB of Q and 131 KB of output or 262 KB of partial sums), a merge 5 to 30.
// 4 trees of 16 heads over 256 keys: 20 us; 64 single tokens over 1024-8192: 79-83, 4.1-4.3 TB/s; 128
// trees: 172-180; 61 trees of 128 heads: 203-213, 640-670 TFLOP/s; 16 long requests of 64 heads:
// 645-720, 0.99-1.10 PFLOP/s (over several cards, whose clocks differ).  Of the 512 registers a lane, 56
// values more are in scratch memory and 106 scalars in lanes: reloaded where a unit is entered and left, not
// in the loops over its tiles.
#include "attn_core.h"

namespace echo {
namespace {

constexpr int kLC = ECHO_LATENT_DIM, kLRow = ECHO_LATENT_DIM + ECHO_LATENT_ROPE_DIM;
constexpr int kLRowBytes = kLRow * 2;          // 1152
constexpr int kLWaves = 4;
constexpr int kLThreads = kLWaves * kWave;
constexpr int kLRows = 128;                    // rows of a unit
constexpr int kLSteps = kLRow / 32;            // products along a row of K
constexpr int kLRestRows = 32;                 // up to here a unit's weights are kept in two numbers
// A tile in LDS: nine blocks (64 dims) of 32 rows x 128 bytes.  The 16-byte chunk c of row r
// is at chunk position c ^ f(r), with bits 3, (2 xor 3), 1 of r as bits 0, 1, 2 of f.  A 16-byte
// read goes in phases of 16 lanes, which are not neighbours (of the first 32: 0-3, 12-15,
// 20-23, 24-27, then the others): eight rows at one chunk of K and eight at its neighbour,
// which f puts into 16 different sixteenths of the banks (with bits 2, 3, 1 of r every
// phase took twice as long); so it does the four rows of which half a wave's transposed
// V read takes four chunks each.
constexpr int kLBlock = kTileKeys * 128;       // 4 KB
// Four slots for the blocks that hold values (a tile is scored a step before its values are
// taken, and two more are on their way), three for the block that only the scores see.
constexpr int kLSlots = 4, kLRopeSlots = 3;
constexpr int kLSlot = 8 * kLBlock;
constexpr int kLProb = kLRows * kTileKeys * 2; // the weights of a tile
constexpr int kLRopeAt = kLSlots * kLSlot, kLProbAt = kLRopeAt + kLRopeSlots * kLBlock;
constexpr int kLStatsAt = kLProbAt + 2 * kLProb;
// (factors [2][128], flags [2][4 waves], inverse sums [128])
constexpr int kLFlagsAt = kLStatsAt + 2 * kLRows * 4, kLInvAt = kLFlagsAt + 16;
constexpr int kLLds = kLInvAt + kLRows * 4;
static_assert(kLLds <= 160 * 1024, "gfx950 LDS per CU");
constexpr int kLOwnPages = 512;                // block tables up to this wide are checked in place

// Costs, in halves of a microsecond: of a tile of a unit with more than 64 rows, of one with fewer; of
// entering such a unit (its rows of Q, its first tiles, its output); the smallest of a
// range, which is a power of two and no smaller than a tile's, so that every range within
// a unit has a tile.
// (Entering at 32 and 56 instead of 40: 61 trees of 128 heads 219 and 215 us for 212.  Tiles at
// 5 : 3 and 8 : 7 instead of 4 : 3: 128 trees of 16 heads 181 and 183 us for 177, long
// requests 740 and 702 for 692.  Smallest ranges of 4 and 16 instead of 8: four
// trees 30.0 and 29.6 us for 28.4.)
constexpr int kLCost4 = 4, kLCost2 = 3, kLEnter4 = 40, kLEnter2 = 16;
constexpr int kLMinShift = 3;
static_assert((1 << kLMinShift) >= kLCost4, "a tile in every range");

// Partial sums per round trip (2.5 us: another XCD wrote them).  Against four, and twice the dims a
// thread: 28.4 to 30.4 us for four trees, 81.3 to 82.8 for 64 single tokens, 212 to 211 for
// 61 trees of 128 heads.
constexpr int kLParts = 8;
// What a round trip costs.  With fewer and larger ranges where that saves more of them: one token of 20 heads over
// 8000 keys 33.6 us for 41.5, two of 128 heads over 6000 41.2 for 49.8, six of 16 over 5000 33.6 for 38.8.
constexpr int kLTrip = 5;
constexpr int kLTwo = 64;  // the smallest range whose units are taken out of order
constexpr int kLMerge = 4, kLMergeRows = 5;  // of a merge, and of 5 x 128 rows of parts, 2.6 MB written and read


typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) uint4v lds_uint4_t;
typedef __attribute__((address_space(3))) uint2v lds_uint2_t;
typedef __attribute__((address_space(3))) float lds_float_t;
typedef __attribute__((address_space(3))) uint32_t lds_uint_t;
typedef __attribute__((address_space(3))) uint8_t lds_byte_t;
typedef __attribute__((address_space(3))) int32_t lds_int_t;
typedef __attribute__((address_space(3))) char lds_char_t;
__device__ __forceinline__ lds_char_t* lds_at(uint32_t x) { return (lds_char_t*)(uintptr_t(x)); }

__host__ __device__ __forceinline__ int l_swz(int row) {
  return (((row >> 1) & 1) << 2) | ((((row >> 2) ^ (row >> 3)) & 1) << 1) | ((row >> 3) & 1);
}

struct LatArgs {
  const uint16_t* q;
  const uint16_t* latent_new;
  const uint16_t* pages;
  const int32_t* block_table;
  const int32_t* prefix_len;
  const int32_t* q_offsets;
  const uint32_t* tree_mask;
  long long num_pages;
  int page_shift, max_pages, W, R, max_rows, hq;
  int chunks;  // flags of latent_pages per request, 0: the workgroups check
  float scale2;
  uint16_t* out;
  float* lse;
  int32_t* status;
};

// A unit whose partial sums have to be merged: those of ranges g - 1, g, ... (parts of them),
// in the record of range g.
struct LatCut {
  int32_t parts, rows;
  int64_t row;  // the first, of all rows of q
};

struct LatWs {
  LatCut* cuts;    // [G]
  int32_t* bad;    // [R][chunks] flags of latent_pages
  float* part_ml;  // [G][2][128][4]: max, sum, sum of the weights used
  float* part_o;   // [G][2][4][128][32][4]: 4 dims of each of 32 rows, 128 times, for four row tiles
};

__host__ inline int l_page_chunks(int max_pages) {
  return max_pages <= kLOwnPages ? 0 : (max_pages + kPageChunk - 1) / kPageChunk;
}

__host__ inline LatWs l_layout(void* base, int R, int max_pages, int G, size_t* bytes) {
  char* p = static_cast<char*>(base);
  LatWs w;
  w.cuts = reinterpret_cast<LatCut*>(p);
  p += al(size_t(G) * sizeof(LatCut));
  w.bad = reinterpret_cast<int32_t*>(p);
  p += al(size_t(R) * size_t(l_page_chunks(max_pages)) * 4);
  w.part_ml = reinterpret_cast<float*>(p);
  p += al(size_t(G) * 2 * kLRows * 4 * sizeof(float));
  w.part_o = reinterpret_cast<float*>(p);
  p += al(size_t(G) * 2 * kLRows * kLC * sizeof(float));
  if (bytes != nullptr) *bytes = size_t(p - static_cast<char*>(base));
  return w;
}

// Pages of a request's prefix, or -1 if its length does not fit its table row.
__device__ __forceinline__ int l_prefix_pages(long long P, const LatArgs& a) {
  if (P < 0 || P > ((long long)a.max_pages << a.page_shift)) return -1;
  return int((P + (1 << a.page_shift) - 1) >> a.page_shift);
}

__global__ __launch_bounds__(kPageChunk) void latent_pages_kernel(LatArgs a, int32_t* bad_flags) {
  const int c = blockIdx.x, r = blockIdx.y;
  const int np = l_prefix_pages(a.prefix_len[r], a);
  const int e = c * kPageChunk + int(threadIdx.x);
  int bad = 0;
  if (e < np) {
    const int pg = a.block_table[size_t(r) * size_t(a.max_pages) + size_t(e)];
    bad = pg < 0 || pg >= a.num_pages;
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) bad_flags[size_t(r) * gridDim.x + c] = bad;
}

// ---------------------------------------------------------------- plan ----
// A request: its units are `full` of 2^us rows (128 or 64) and, if there are rows left, one more.
struct LatLook {
  int q0, n, P;
  bool ok;
  __device__ __forceinline__ int rows(const LatArgs& a) const { return n * a.hq; }
  __device__ __forceinline__ int tree_tiles() const { return (n + kTileKeys - 1) / kTileKeys; }
  __device__ __forceinline__ int tiles() const {
    return tree_tiles() + int((unsigned(P) + kTileKeys - 1) / kTileKeys);
  }
};
__device__ __forceinline__ LatLook l_look(const LatArgs& a, int r) {
  LatLook x;
  const int q0 = a.q_offsets[r], q1 = a.q_offsets[r + 1], P = a.prefix_len[r];
  x.ok = q0 >= 0 && q1 >= q0 && q1 <= a.max_rows && l_prefix_pages(P, a) >= 0;
  x.q0 = q0;
  x.n = x.ok ? q1 - q0 : 0;
  x.P = x.ok ? P : 0;
  return x;
}
__device__ __forceinline__ int l_tile_cost(int rows) { return rows > kLRows / 2 ? kLCost4 : kLCost2; }
__device__ __forceinline__ int l_enter_cost(int rows) { return rows > kLRows / 2 ? kLEnter4 : kLEnter2; }
__device__ __forceinline__ int l_unit_cost(int tiles, int rows) {
  return l_enter_cost(rows) + tiles * l_tile_cost(rows);  // (tiles < 2^27)
}
// Costs are summed in 32 bits and saturate; a batch of 2^31 or more (four seconds) is refused.
__device__ __forceinline__ uint32_t l_cost(const LatArgs& a, const LatLook& x, int us) {
  if (x.n == 0) return 0;
  const int rows = x.rows(a), rest = rows & ((1 << us) - 1);
  const uint64_t c = uint64_t(uint32_t(rows >> us)) * uint32_t(l_unit_cost(x.tiles(), 1 << us)) +
                     uint32_t(rest > 0 ? l_unit_cost(x.tiles(), rest) : 0);
  return (c >> 32) != 0 ? 0xFFFFFFFFu : uint32_t(c);
}
__device__ __forceinline__ int l_units(const LatArgs& a, const LatLook& x, int us) {
  return (x.rows(a) + (1 << us) - 1) >> us;
}
struct AddSatOp {
  __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return __builtin_elementwise_add_sat(a, b); }
};

// Ranges 0 .. 2^shift - 1 of [0, total).
struct LatRanges {
  int total, shift;
  __device__ __forceinline__ int first(int g) const { return int((uint64_t(uint32_t(total)) * uint32_t(g)) >> shift); }
  // The range that holds cost x.
  __device__ __forceinline__ int range_of(int x) const {
    const int n = 1 << shift;
    int g = min(int(float(x) * float(n) * __builtin_amdgcn_rcpf(float(total))), n - 1);
    while (g > 0 && first(g) > x) --g;
    while (g + 1 < n && first(g + 1) <= x) ++g;
    return g;
  }
};
// The first tile that starts at cost x or later, of T tiles of cost c (kLCost4 or kLCost2) from cost 0 on.
__device__ __forceinline__ int l_tile_at(int x, int c, int T) {
  if (x <= 0) return 0;
  if (x > (T - 1) * c) return T;
  return c == kLCost4 ? (x + kLCost4 - 1) / kLCost4 : (x + kLCost2 - 1) / kLCost2;
}

// The lane, formed where it is used: what would be kept from it over a step is reloaded from
// memory, behind every copy in flight.
__device__ __forceinline__ int l_lane() {
  int x = int(__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)));
  asm volatile("" : "+v"(x));
  return x;
}

__device__ __forceinline__ int l_opaque(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
// A value that all lanes have, in a scalar register (the compiler, which knows that it is uniform, would
// leave what vector instructions computed in vector ones, and all that follows from it).
__device__ __forceinline__ int l_scalar(int x) { return __builtin_amdgcn_readfirstlane(l_opaque(x)); }

// Whether a thread sees a page of a request that is not in the pool (for an or over all threads).
__device__ __forceinline__ int l_pages_bad(const LatArgs& a, const LatWs& ws, int r, int P) {
  const int np = l_prefix_pages(P, a), tid = wave_id() * kWave + l_lane();
  int bad = 0;
  if (a.chunks == 0) {
    static_assert(kLOwnPages <= 2 * kLThreads, "two entries a thread, in one round trip");
    const int32_t* e = a.block_table + size_t(r) * size_t(a.max_pages);
    int v[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (tid + k * kLThreads < np) v[k] = e[tid + k * kLThreads];
#pragma unroll
    for (int k = 0; k < 2; ++k) bad |= v[k] < 0 || (v[k] > 0 && v[k] >= a.num_pages);
  } else {
    const int32_t* e = ws.bad + size_t(r) * size_t(a.chunks);
    for (int i = tid; i < (np + kPageChunk - 1) / kPageChunk; i += kLThreads) bad |= e[i] != 0;
  }
  return bad;
}

// ---------------------------------------------------------------- main ----
// Piece B (of nine) of the copy of a wave's eight rows of a tile: 1 KB, from base + off + 128 B to
// LDS address lds + 4096 B (B < 8) or rope.  The instruction's offset moves both addresses.
// In inline assembly because the compiler would wait for every copy in flight before each
// LDS read.  The compiler does not see a load here: M0, the LDS address, needs a wait state before
// it, and scalars that a vector instruction wrote (base, by a lane's read) five.
constexpr int kLCopies = 9;  // loads of a wave per tile
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (M0 is reserved: nothing of the compiler's is kept in it)
template <int B>
__device__ __forceinline__ void l_copy(uint32_t lds, uint32_t rope, uint64_t base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2 offset:%3"
               :
               : "s"(B < 8 ? lds + uint32_t(B * (kLBlock - 128)) : rope - 8 * 128u), "v"(off), "s"(base), "n"(B * 128)
               : "memory", "m0");
}
#pragma clang diagnostic pop

struct LatUnit {
  int q0, n, P, r, row0, rows, tree_tiles;
  int w;  // the wave, in a scalar register (formed in a step, the thread's number is reloaded from memory)
};

// The addresses of 64 tiles of a unit, tile at + i in lane i: one vector of loads, where scalar ones
// would be waited for with every LDS read.
struct LatTable {
  uint32_t lo, hi;
  int at;
};
__device__ __forceinline__ void l_fill(LatTable& tb, const LatArgs& a, const LatUnit& u, int t) {
  const int lane = l_lane();
  tb.at = t;
  uint64_t base;
  if (t + lane < u.tree_tiles) {
    base = reinterpret_cast<uint64_t>(a.latent_new) + uint64_t(u.q0 + (t + lane) * kTileKeys) * kLRowBytes;
  } else {
    const long long key = (long long)(t + lane - u.tree_tiles) * kTileKeys;
    int page = 0;
    if (key < u.P) page = a.block_table[size_t(u.r) * size_t(a.max_pages) + size_t(key >> a.page_shift)];
    if (page < 0 || page >= a.num_pages) page = 0;  // (read before the pages are checked)
    const uint64_t row = (uint64_t(uint32_t(page)) << a.page_shift) + uint32_t(key & ((1 << a.page_shift) - 1));
    base = reinterpret_cast<uint64_t>(a.pages) + row * kLRowBytes;
  }
  tb.lo = uint32_t(base);
  tb.hi = uint32_t(base >> 32);
  asm volatile("" : "+v"(tb.lo), "+v"(tb.hi));  // (waited for here, not where every step would)
}

// What the copies of a tile take: tile t of a unit, the n-th that its workgroup copies.
struct LatCopy {
  uint64_t base;
  uint32_t off, lds, rope;
  template <int B>
  __device__ __forceinline__ void piece() const { l_copy<B>(lds, rope, base, off); }
};
__device__ __forceinline__ LatCopy l_tile(LatTable& tb, const LatArgs& a, const LatUnit& u, int t, int n,
                                          uint32_t smem) {
  const int w = u.w;
  LatCopy c;
  if (t >= tb.at + kWave) l_fill(tb, a, u, t);
  c.base = uint64_t(uint32_t(__builtin_amdgcn_readlane(int(tb.lo), t - tb.at))) |
           (uint64_t(uint32_t(__builtin_amdgcn_readlane(int(tb.hi), t - tb.at))) << 32);
  const int tn = t < u.tree_tiles ? u.n - t * kTileKeys : u.P - (t - u.tree_tiles) * kTileKeys;
  const int lane = l_lane();
  const int key = 8 * w + (lane >> 3);
  // (rows past the tile's keys: the last one again, so that nothing unwritten is multiplied)
  c.off = uint32_t(min(key, tn - 1) * kLRowBytes + (((lane & 7) ^ l_swz(key)) << 4));
  const uint32_t at = smem + uint32_t(w * 1024);
  c.lds = __builtin_amdgcn_readfirstlane(at + uint32_t(n & (kLSlots - 1)) * kLSlot);
  c.rope = __builtin_amdgcn_readfirstlane(at + kLRopeAt + (unsigned(n) % kLRopeSlots) * kLBlock);
  return c;
}
__device__ __forceinline__ void l_send(LatTable& tb, const LatArgs& a, const LatUnit& u, int t, int n, uint32_t smem) {
  const LatCopy c = l_tile(tb, a, u, t, n, smem);
  c.piece<0>();
  c.piece<1>();
  c.piece<2>();
  c.piece<3>();
  c.piece<4>();
  c.piece<5>();
  c.piece<6>();
  c.piece<7>();
  c.piece<8>();
}

__device__ __forceinline__ float quad_max(float v) {  // over the four lanes of a row
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

__device__ __forceinline__ void l_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// acc += A B with acc in accumulation registers.  In inline assembly because 128 rows x 128 dims
// are all 256 of them, and the compiler holds other products' results there too, or
// copies.  The compiler does not know the wait states around it: one after a vector
// instruction that writes an operand, before; those before acc is read, l_settle.
__device__ __forceinline__ void l_mfma(floatx16& acc, bf16x8 x, bf16x8 y) {
  asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(x), "v"(y));
}
__device__ __forceinline__ void l_settle(floatx16& acc) { asm volatile("s_nop 15\n\ts_nop 15" : "+a"(acc)); }

#define ECHO_FENCE() __builtin_amdgcn_sched_barrier(0)

// A wave's state over a unit.
template <int QR>
struct LatState {
  bf16x8 q[QR][kLSteps];   // row l16 of each 16-row tile, dims 32 ks + 8 quad ..
  floatx16 o[2 * QR][4];   // O^T: row tile, dims 128 w + 32 ct + 8 (r >> 2) + 4 h + (r & 3)
  float m[QR], l[QR], lq[QR];
};

// One step: the scores of tile t + 1 (kScores), which is the n + 1-th copied, and the values of
// tile t (kValues), the n-th; copies for tile t + 3.  A tile's 16-key groups x 32-dim
// columns are eight groups of products with V: two are taken between the next tile's scores,
// the others beside its softmax.  kRest: rows 32 .. 63 are rows 0 .. 31 once more, of whose
// weights waves 2 and 3 take p - bf16(p).
template <int QR, bool kRest, bool kScores, bool kValues>
__device__ __forceinline__ void l_step(LatState<QR>& st, LatTable& tb, const LatArgs& a, const LatUnit& u, int t,
                                       int t1, int n, uint32_t smem, uint32_t ka, uint32_t va, uint32_t pw) {
  constexpr int RT = 2 * QR;  // 32-row tiles of the unit
  constexpr int kAhead = 2;   // steps of 32 dims that K's reads are ahead of its products
  const int w = u.w;
  const uint32_t rest = 0u - uint32_t(w >> 1);  // all bits in waves 2 and 3
  // tile t + 1 has landed (t + 2 may be behind it), the weights of t are written
  if (kScores) {
    if (t + 2 < t1) wait_vm<kLCopies>();
    else wait_vm<0>();
  }
  wait_lds();
  l_barrier();

  const uint32_t now = smem + uint32_t(n & (kLSlots - 1)) * kLSlot;
  const uint32_t next = smem + uint32_t((n + 1) & (kLSlots - 1)) * kLSlot;
  const uint32_t rope = smem + kLRopeAt + (unsigned(n + 1) % kLRopeSlots) * kLBlock;
  const uint32_t buf = uint32_t(n & 1), buf1 = buf ^ 1u;
  const uint32_t kb = next + ka, rb = rope + ka;
  // V's addresses, kept: formed at each read they were 40 instructions a step, 2.5% of 61 trees of 128 heads.
  uint32_t vat[2][2];
#pragma unroll
  for (int k = 0; k < 4; ++k) vat[k >> 1][k & 1] = uint32_t(l_opaque(int((now + va) ^ uint32_t(((k >> 1) << 6) | ((k & 1) * 48)))));
  const uint32_t pb = smem + kLProbAt + buf * kLProb + uint32_t(l_lane() * 16);
  bf16x8 kf[kAhead + 1][2], vf[2], pf[RT];
  floatx4 s[QR][2];
  const auto read_k = [&](int ks) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
      kf[ks % (kAhead + 1)][kt] = __builtin_bit_cast(
          bf16x8, ks < 16 ? *(lds_uint4_t*)(lds_at(kb ^ uint32_t((ks & 1) << 6)) + (ks >> 1) * kLBlock + kt * 2048)
                          : *(lds_uint4_t*)(lds_at(rb ^ uint32_t((ks & 1) << 6)) + kt * 2048));
  };
  const auto read_v = [&](int g) {  // keys 16 (g / 4) .., dims 32 (g % 4) .. of the wave's
    const int kg = g >> 2, ct = g & 3;
    shortx4 v[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
      v[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_shortx4_t*)(lds_at(vat[ct & 1][k]) + (ct >> 1) * kLBlock + kg * 2048 + k * 1024));
    vf[g & 1] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };
  const auto read_p = [&](int kg, int rt) {
    pf[rt] = __builtin_bit_cast(bf16x8, *(lds_uint4_t*)(lds_at(pb) + rt * 2048 + kg * 1024));
  };
  const auto group = [&](int g) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) l_mfma(st.o[kRest ? 0 : rt][g & 3], vf[g & 1], pf[rt]);
  };

  uint32_t flags = 0;  // (a byte for each wave)
  if (kValues) flags = *(lds_uint_t*)lds_at(smem + kLFlagsAt + 4 * buf);
  const auto rescale = [&] {  // O is scaled where a reference was raised
    flags = uint32_t(__builtin_amdgcn_readfirstlane(int(flags)));
    if (flags == 0) return;
#pragma unroll
    for (int rt = 0; rt < (kRest ? 1 : RT); ++rt) {
      const uint32_t f = QR == 2 ? flags >> (8 * rt) : flags >> (16 * rt);
      if ((f & (QR == 2 ? 0xFFu : 0xFFFFu)) != 0) {
        const int lane = l_lane();
        float alpha = *(lds_float_t*)lds_at(smem + kLStatsAt + buf * (kLRows * 4) + uint32_t((32 * rt + (lane & 31)) * 4));
        if (QR == 1) alpha = ((f >> (8 * ((lane >> 4) & 1))) & 0xFFu) != 0 ? alpha : 1.0f;
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) {
          l_settle(st.o[rt][ct]);
          st.o[rt][ct] *= alpha;
        }
      }
    }
  };
  const auto read_first = [&] {
    read_v(0);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) read_p(0, rt);
  };
  const bool send = kScores && kValues && t + 3 < t1;
  LatCopy copy = {};
  // S^T: keys 16 kt + 4 quad + r of row l16
  if (kScores) {
#pragma unroll
    for (int ks = 0; ks < kAhead; ++ks) read_k(ks);
    if (kValues) rescale();
#pragma unroll
    for (int i = 0; i < QR; ++i) s[i][0] = s[i][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < kLSteps; ++ks) {
      if (ks + kAhead < kLSteps) read_k(ks + kAhead);
      if (kValues && (ks == 8 || ks == 13)) {
        const int g = ks == 8 ? 0 : 1;
        read_v(g + 1);
        ECHO_FENCE();
        group(g);
      }
      ECHO_FENCE();
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < QR; ++i)
          s[i][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[ks % (kAhead + 1)][kt], st.q[i][ks], s[i][kt], 0, 0, 0);
      ECHO_FENCE();
      // In the products' shadow: the copies of tile t + 3 (in two lots; one to a step of 32 dims, nine of them, or
      // all in one cost 1-2% of the cycles more), the first operands of the products with V.
      if (kValues) {
        if (ks == 0 && send) copy = l_tile(tb, a, u, t + 3, n + 3, smem);
        if (send) {
          if (ks == 2) {
            copy.piece<0>();
            copy.piece<1>();
            copy.piece<2>();
            copy.piece<3>();
            copy.piece<4>();
          }
          if (ks == 4) {
            copy.piece<5>();
            copy.piece<6>();
            copy.piece<7>();
            copy.piece<8>();
          }
        }
        if (ks == 5) read_first();
      }
    }
  } else if (kValues) {
    rescale();
    read_first();
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      read_v(g + 1);
      ECHO_FENCE();
      group(g);
      ECHO_FENCE();
    }
  }
  const int tt = t + 1;
  const bool tree = tt < u.tree_tiles;
  const int tn = tree ? u.n - tt * kTileKeys : u.P - (tt - u.tree_tiles) * kTileKeys;
  float top[QR], neg_m[QR];
  if (kValues) {
    read_v(3);
    ECHO_FENCE();
    l_mfma(st.o[0][2], vf[0], pf[0]);
    ECHO_FENCE();
  }
  if (kScores && (tree || tn < kTileKeys)) {  // masks: the tree's words, the prefix's last tile
#pragma unroll
    for (int i = 0; i < QR; ++i) {
      uint32_t word = 0xFFFFFFFFu;
      if (tree) {
        const int slot = *(lds_int_t*)lds_at(smem + kLInvAt + uint32_t((16 * (QR * w + i) + (l_lane() & 15)) * 4));
        word = tt < a.W ? a.tree_mask[size_t(slot) * a.W + tt] : 0u;
      }
      if (tn < kTileKeys) word &= (1u << tn) - 1u;
      word >>= 4 * (l_lane() >> 4);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          s[i][kt][r] = ((word >> (16 * kt + r)) & 1u) ? s[i][kt][r] : -__builtin_inff();
    }
  }
  const auto max_of = [&](int i) {
    top[i] = fmaxf(fmaxf(fmaxf(s[i][0][0], s[i][0][1]), fmaxf(s[i][0][2], s[i][0][3])),
                   fmaxf(fmaxf(s[i][1][0], s[i][1][1]), fmaxf(s[i][1][2], s[i][1][3]))) * a.scale2;
  };
  if (kValues) {
#pragma unroll
    for (int x = 1; x < 2 * RT; ++x) {  // the rest of group 2, and group 3
      const int g = 2 + x / RT, rt = x % RT;
      if (x == RT) read_v(4);
      ECHO_FENCE();
      l_mfma(st.o[kRest ? 0 : rt][g], vf[g & 1], pf[rt]);
      ECHO_FENCE();
      if (g == 3) read_p(1, rt);
      if (kScores && x <= QR) max_of(x - 1);
    }
  } else if (kScores) {
#pragma unroll
    for (int i = 0; i < QR; ++i) max_of(i);
  }
  bool raised = false;
  if (kScores) {
    // The reference is raised only when a logit (in powers of two) exceeds it by more than 8: weights stay <= 2^8.
    bool up = false;
#pragma unroll
    for (int i = 0; i < QR; ++i) up |= top[i] > st.m[i] + kRescaleSlack;
    raised = __ballot(up) != 0ull;
    if (raised) {
#pragma unroll
      for (int i = 0; i < QR; ++i) {
        const float mt = quad_max(top[i]);
        const bool grow = mt > st.m[i] + kRescaleSlack;
        const float alpha = grow ? __builtin_amdgcn_exp2f(st.m[i] - mt) : 1.0f;  // 0 from -inf
        st.l[i] *= alpha;
        st.lq[i] *= alpha;
        st.m[i] = grow ? mt : st.m[i];
        const int lane = l_lane();
        if (lane < 16)
          *(lds_float_t*)lds_at(smem + kLStatsAt + buf1 * (kLRows * 4) + uint32_t((16 * (QR * w + i) + lane) * 4)) = alpha;
      }
    }
#pragma unroll
    for (int i = 0; i < QR; ++i) neg_m[i] = st.m[i] == -__builtin_inff() ? 0.0f : -st.m[i];
  }
  // Weights 2 (p % 2) and the next of tile p / 2 % 2 of row tile p / 4: the exponentials of a pair beside
  // one product, its sums and roundings beside the next, so that neither waits for the other.
  float x0 = 0.0f, x1 = 0.0f;
  uint32_t half = 0;
  const auto weigh = [&](int p) {
    const int i = p >> 2, kt = (p >> 1) & 1, r = 2 * (p & 1);
    x0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][kt][r], a.scale2, neg_m[i]));
    x1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][kt][r + 1], a.scale2, neg_m[i]));
  };
  const auto take = [&](int p) {
    const int i = p >> 2, kt = (p >> 1) & 1;
    st.l[i] += x0 + x1;
    uint32_t xy = pack_bf16x2(x0, x1);
    if (kRest) {  // (the differences are exact; the sum is st.l)
      const uint32_t sub = xy & rest;
      xy = pack_bf16x2(x0 - __uint_as_float(sub << 16), x1 - __uint_as_float(sub & 0xFFFF0000u));
    } else {
      st.lq[i] = add_bf16x2(xy, st.lq[i]);
    }
    if ((p & 1) == 0) half = xy;
    else *(lds_uint2_t*)(lds_at(pw + buf1 * kLProb) + kt * 1024 + i * 256) = uint2v{half, xy};
  };
  const auto tell = [&] {  // (before the first values O is 0)
    if (l_lane() == 0) *(lds_byte_t*)lds_at(smem + kLFlagsAt + 4 * buf1 + uint32_t(w)) = kValues && raised ? 1 : 0;
  };
  if (kValues) {
#pragma unroll
    for (int x = 0; x < 4 * RT; ++x) {
      const int g = 4 + x / RT, rt = x % RT;
      if (rt == 0 && g < 7) read_v(g + 1);
      ECHO_FENCE();
      l_mfma(st.o[kRest ? 0 : rt][g & 3], vf[g & 1], pf[rt]);
      ECHO_FENCE();
      if (kScores) {
        if ((x & 1) == 0) weigh(x >> 1);
        else take(x >> 1);
      }
    }
    ECHO_FENCE();
    if (kScores) tell();
  } else if (kScores) {
#pragma unroll
    for (int p = 0; p < 4 * QR; ++p) {
      weigh(p);
      take(p);
    }
    tell();
  }
}

// Tiles [t0, t1) of a unit, then its output (whole) or partial sums (part).  QR: 16-row tiles of
// a wave's part of Q; the unit has up to 64 QR rows.  check: the request's pages have not
// been looked at yet; false if they are not all in the pool, and nothing is written.
template <int QR, bool kRest>
__device__ __forceinline__ bool l_segment(const LatArgs& a, const LatWs& ws, const LatUnit& u, int t0,
                                          int t1, bool whole, size_t part, bool check, uint32_t smem) {
  constexpr int OT = kRest ? 1 : 2 * QR;  // 32-row tiles of O
  const int w = u.w;
  const size_t first = size_t(u.q0) * a.hq + size_t(u.row0);  // the unit's first row of q

  // Page ids first, then the first tiles' copies, then Q, of which there is most: loads return in
  // order.
  const int bad = check ? l_pages_bad(a, ws, u.r, u.P) : 0;
  LatTable tb;
  l_fill(tb, a, u, t0);
  l_send(tb, a, u, t0, 0, smem);
  if (t0 + 1 < t1) l_send(tb, a, u, t0 + 1, 1, smem);
  LatState<QR> st;
#pragma unroll
  for (int i = 0; i < QR; ++i) {  // (rows past the last: the last again)
    const int lane = l_lane();
    const int row = min((16 * (QR * w + i) + (lane & 15)) & (kRest ? 31 : 127), u.rows - 1);
    const uint16_t* p = a.q + (first + row) * kLRow + 8 * (lane >> 4);
#pragma unroll
    for (int ks = 0; ks < kLSteps; ++ks) st.q[i][ks] = as_bf16x8(*reinterpret_cast<const uint4*>(p + 32 * ks));
    // (for the tree's masks; the sums take the place)
    if (lane < 16) *(lds_int_t*)lds_at(smem + kLInvAt + uint32_t((16 * (QR * w + i) + lane) * 4)) = u.q0 + (u.row0 + row) / a.hq;
    st.m[i] = -__builtin_inff();
    st.l[i] = st.lq[i] = 0.0f;
  }
  if (check && __builtin_amdgcn_readfirstlane(__syncthreads_or(bad)) != 0) {
    wait_vm<0>();  // (nothing is on its way to LDS)
    l_barrier();
    return false;
  }
#pragma unroll
  for (int rt = 0; rt < OT; ++rt)
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) st.o[rt][ct] = floatx16{};
  // LDS offsets in a tile
  const int lane = l_lane(), l16 = lane & 15, quad = lane >> 4, h = lane >> 5;
  const uint32_t ka = uint32_t(l16 * 128 + ((quad ^ l_swz(l16)) << 4));
  const int vkey = 4 * h + (l16 >> 2);
  const uint32_t vchunk = uint32_t((2 * (quad & 1) + ((l16 & 3) >> 1)) ^ l_swz(vkey));
  const uint32_t va = uint32_t(2 * w * kLBlock + vkey * 128 + ((l16 & 1) << 3)) + (vchunk << 4);
  const uint32_t pw = smem + kLProbAt + uint32_t((QR == 2 ? w : w >> 1) * 2048 +
                                                 ((QR == 2 ? 0 : 16 * (w & 1)) + l16) * 16 + (quad & 1) * 512 +
                                                 (quad >> 1) * 8);
  l_step<QR, kRest, true, false>(st, tb, a, u, t0 - 1, t1, -1, smem, ka, va, pw);
  if (t0 + 2 < t1) l_send(tb, a, u, t0 + 2, 2, smem);
  int t = t0;
#pragma unroll 1
  for (; t + 1 < t1; ++t) l_step<QR, kRest, true, true>(st, tb, a, u, t, t1, t - t0, smem, ka, va, pw);
  l_step<QR, kRest, false, true>(st, tb, a, u, t, t1, t - t0, smem, ka, va, pw);
#pragma unroll
  for (int rt = 0; rt < OT; ++rt)
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) l_settle(st.o[rt][ct]);

  // the sums of a row are its wave's; every wave needs their inverses
#pragma unroll
  for (int i = 0; i < QR; ++i) {
    const float L = quad_sum(st.l[i]), Lq = kRest ? L : quad_sum(st.lq[i]);
    const int lane = l_lane();
    const int row = 16 * (QR * w + i) + (lane & 15);
    if (lane < 16) {
      *(lds_float_t*)lds_at(smem + kLInvAt + uint32_t(row * 4)) = Lq > 0.0f ? 1.0f / Lq : 0.0f;
      if (row < u.rows) {
        if (!whole)
          *reinterpret_cast<floatx4*>(ws.part_ml + (part * kLRows + row) * 4) = floatx4{st.m[i], L, Lq, 0.0f};
        else if (a.lse != nullptr)
          a.lse[first + row] = L > 0.0f ? (st.m[i] + log2f(L)) * kLn2 : -__builtin_inff();
      }
    }
  }
  wait_lds();
  l_barrier();  // (the slots are free too)
  if (whole) {
    // O^T through the wave's own slot: 32 rows x 256 bytes, 16-byte chunk c of row r at c ^ (r & 15), so
    // that a row's 256 bytes go out in one piece
    const uint32_t own = smem + uint32_t(w) * kLSlot;
#pragma unroll
    for (int rt = 0; rt < OT; ++rt) {
      const int lane = l_lane(), rl = lane & 31, h = lane >> 5;
      const float inv = *(lds_float_t*)lds_at(smem + kLInvAt + uint32_t((32 * rt + rl) * 4));
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *(lds_uint2_t*)lds_at(own + uint32_t(rt * 8192 + rl * 256 + (((4 * ct + (r >> 2)) ^ (rl & 15)) << 4) + 8 * h)) =
              uint2v{pack_bf16x2(st.o[rt][ct][r] * inv, st.o[rt][ct][r + 1] * inv),
                     pack_bf16x2(st.o[rt][ct][r + 2] * inv, st.o[rt][ct][r + 3] * inv)};
    }
    const int lane = l_lane(), l16 = lane & 15, quad = lane >> 4;
    uint16_t* po = a.out + first * kLC + 128 * w + 8 * l16;
#pragma unroll
    for (int k = 0; k < 8 * OT; ++k) {
      const int row = 4 * k + quad;
      const uint4v x = *(lds_uint4_t*)lds_at(own + uint32_t(row * 256 + ((l16 ^ (row & 15)) << 4)));
      if (row < u.rows) *reinterpret_cast<uint4v*>(po + size_t(row) * kLC) = x;
    }
    wait_lds();
    l_barrier();  // (the next unit's tiles take the slots)
  } else {
#pragma unroll
    for (int rt = 0; rt < OT; ++rt) {
      const int lane = l_lane(), h = lane >> 5;
      if (32 * rt + (lane & 31) >= u.rows) continue;
      float* po = ws.part_o + ((part * 4 + rt) * 128 + 32 * w + h) * 128 + (lane & 31) * 4;
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *reinterpret_cast<floatx4*>(po + (8 * ct + (r >> 1)) * 128) =
              floatx4{st.o[rt][ct][r], st.o[rt][ct][r + 1], st.o[rt][ct][r + 2], st.o[rt][ct][r + 3]};
    }
  }
  return true;
}

__global__ __launch_bounds__(kLThreads) __attribute__((amdgpu_waves_per_eu(1, 1))) void latent_main_kernel(
    LatArgs a, LatWs ws) {
  __shared__ __attribute__((aligned(1024))) char smem[kLLds];
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  int wid = wave_id();
  asm volatile("" : "+s"(wid));
  const int nwg = int(gridDim.x);
  // every thread counts the costs and units of K requests, with units of 128 rows and of 64
  uint32_t* s_start = reinterpret_cast<uint32_t*>(smem);  // [threads]
  uint4* s_sums = reinterpret_cast<uint4*>(smem) + kLThreads / 4;  // [waves]: costs, units
  uint32_t* s_longest = reinterpret_cast<uint32_t*>(s_sums + kLWaves);  // [waves]
  const int K = (a.R + kLThreads - 1) / kLThreads;
  uint32_t mine = 0, mine64 = 0;
  int bits = 0, longest = 0, units = 0, units64 = 0;
  for (int i = 0; i < K; ++i) {
    const int r = tid * K + i;
    if (r >= a.R) break;
    const LatLook x = l_look(a, r);
    if (!x.ok) bits = ECHO_DATA_BAD_OFFSETS;
    mine = AddSatOp{}(mine, l_cost(a, x, 7));
    mine64 = AddSatOp{}(mine64, l_cost(a, x, 6));
    units += l_units(a, x, 7);
    units64 += l_units(a, x, 6);
    if (x.n > 0) longest = max(longest, x.tiles());
  }
  const uint32_t upto = wave_scan(mine, 0u, AddSatOp{}), upto64 = wave_scan(mine64, 0u, AddSatOp{});
  const int upto_n = wave_inclusive_sum(units), upto_n64 = wave_inclusive_sum(units64);
  longest = int(wave_max(uint32_t(longest)));
  if (lane == kWave - 1) {
    s_sums[wid] = make_uint4(upto, upto64, uint32_t(upto_n), uint32_t(upto_n64));
    s_longest[wid] = uint32_t(longest);
  }
  __syncthreads();
  uint32_t before[4] = {}, all[4] = {};
  longest = 0;
#pragma unroll
  for (int v = 0; v < kLWaves; ++v) {
    const uint4 x4 = s_sums[v];
    const uint32_t x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (v < wid) before[k] = AddSatOp{}(before[k], x[k]);
      all[k] = AddSatOp{}(all[k], x[k]);
    }
    longest = max(longest, int(s_longest[v]));
  }
  longest = l_scalar(longest);
  const uint32_t total128 = uint32_t(l_scalar(int(all[0]))), total64 = uint32_t(l_scalar(int(all[1])));
  // Units of 64 rows where entering one of 128 takes longer than its tiles, of which it has two thirds of the
  // other's per row: 4 trees of 16 heads 22.6 us for 27.9, one token of 128 heads 17.9 for 24.7, 40
  // of them over 2000-3000 tokens 65.5 for 69.9; units of 64 rows throughout: 61 trees of
  // 128 heads would have 1.4 times the work.
  const bool small = int(total64 - total128) < (kLEnter4 - kLEnter2) * nwg && int(total64) >= 0;
  const int us = small ? 6 : 7;
  const uint32_t total = small ? total64 : total128;
  if (int(total) < 0) bits = ECHO_DATA_BAD_OFFSETS;  // 2^31 or more
  if (blockIdx.x == 0) wave_status_or(a.status, bits);
  LatRanges ranges;
  ranges.total = max(int(total), 0);
  // as many as there are workgroups, or fewer (powers of two)
  const int most = 31 - __builtin_clz(nwg);
  ranges.shift = most;
  while (ranges.shift > 0 && (ranges.total >> (ranges.shift + kLMinShift)) == 0) --ranges.shift;
  // Fewer where that saves more round trips of the merge than it costs: ranges of twice the size, half the parts.
  const int unit = l_unit_cost(longest, 1 << us);
  while (ranges.shift > 0) {
    const int range = ranges.total >> ranges.shift;
    if (unit <= kLParts * range) break;  // (one round trip)
    const int trips = l_scalar((unit / range + kLParts - 1) / kLParts);
    if (range >= kLTrip * (trips / 2)) break;
    --ranges.shift;
  }
  // Or none is cut, if the longest unit takes no longer than a range with a unit entered in its middle and the
  // merge of what was cut (its start, and the parts' bytes): 116 single tokens over 50-83 keys 18.9 us
  // for 21.5, 16 trees of 11 slots over 65-83 20.1 for 23.7, 30 trees of 32 heads over 26-54 20.1 for 29.1.
  const int n = l_scalar(int(small ? all[3] : all[2])), range = ranges.total >> ranges.shift;
  const int rows_most = int(min((long long)a.max_rows * a.hq, (long long)n << us) >> 7);
  const int merge = l_scalar(kLMerge + (rows_most << ranges.shift) / max(min(n, 1 << 20) * kLMergeRows, 1));
  const bool whole = n > 0 && n <= (1 << most) && unit > range && unit <= range + (small ? kLEnter2 : kLEnter4) + merge;
  if (whole) {
    ranges.total = n;
    ranges.shift = min(32 - __builtin_clz(n), most);
  }
  s_start[tid] = whole ? uint32_t(small ? int(before[3]) + upto_n64 - units64 : int(before[2]) + upto_n - units)
                       : (small ? before[1] + upto64 - mine64 : before[0] + upto - mine);
  __syncthreads();
  // neighbouring ranges, which share requests, run on one XCD (workgroup b is on XCD b % 8)
  int g = blockIdx.x;
  if ((1 << ranges.shift) == nwg && nwg % 8 == 0) g = (g & 7) * (nwg / 8) + (g >> 3);
  if (tid == 0) ws.cuts[g].parts = 0;  // (unless there is one: below, by the same thread)
  if (g >= (1 << ranges.shift) || ranges.total == 0) return;
  const int lo = ranges.first(g), hi = ranges.first(g + 1);
  if (lo >= hi) return;
  // the last thread whose requests start at lo or before, and which of its requests it is
  int th = 0;
#pragma unroll
  for (int v = 0; v < kLWaves; ++v) th += __popcll(__ballot(int(s_start[v * kWave + lane]) <= lo));
  th = __builtin_amdgcn_readfirstlane(th) - 1;
  LatLook x = {};
  int r = th * K + lane;
  if (lane < K && r < a.R) x = l_look(a, r);
  int at;  // where the request's units start
  {
    const int c = whole ? l_units(a, x, us) : int(l_cost(a, x, us));
    const int end = int(s_start[th]) + wave_inclusive_sum(c);
    const int i = __ffsll((unsigned long long)__ballot(end > lo)) - 1;
    r = th * K + i;
    at = __shfl(end - c, i);
    x.q0 = __shfl(x.q0, i);
    x.n = __shfl(x.n, i);
    x.P = __shfl(x.P, i);
  }
  __syncthreads();  // (the tiles take this memory)
  const uint32_t base = __builtin_amdgcn_readfirstlane(uint32_t(reinterpret_cast<uintptr_t>((lds_void_t*)smem)));
  // The unit that the range starts in, if it did before it: last, so that units that start in it, of which a
  // request often has one in each of its ranges, go over the same keys at once (16 long requests read
  // 2.2 GB instead of 3.0, and the clock is higher for it: 666 us for 691; 61 trees of 128 heads
  // 203 for 206).  Only where a request has several units and ranges are long, as it takes time to find out.
  r = l_scalar(r);
  x.q0 = l_scalar(x.q0);
  x.n = l_scalar(x.n);
  x.P = l_scalar(x.P);
  at = l_scalar(at);
  const auto unit_of = [&](const LatLook& y, int y_at, int from) {  // the one that starts at cost `from` or before it
    const int full = y.rows(a) >> us, full_unit = whole ? 1 : l_unit_cost(y.tiles(), 1 << us);
    int j = 0;
    if (from > y_at && full > 0) {
      j = min(int(float(from - y_at) * __builtin_amdgcn_rcpf(float(full_unit))), full);
      while (j > 0 && y_at + j * full_unit > from) --j;
      while (j < full && y_at + (j + 1) * full_unit <= from) ++j;
      j = l_scalar(j);
    }
    return j;
  };
  const LatLook x0 = x;
  const int r0 = r, at0 = at;
  int split = hi;  // where that unit ends
  if (!whole && range >= kLTwo && x0.rows(a) > 1 << us) {
    const int T = x0.tiles(), j = unit_of(x0, at0, lo), rows = min(1 << us, x0.rows(a) - (j << us));
    const int start = at0 + j * l_unit_cost(T, 1 << us);
    if (lo > start + l_enter_cost(rows)) split = l_scalar(min(start + l_unit_cost(T, rows), hi));
  }
  const bool two = split < hi;
#pragma unroll 1
  for (int pass = two ? 0 : 1; pass < 2; ++pass) {
    const int from = pass == 0 ? split : lo, to = pass == 1 && two ? split : hi;
    r = r0;
    x = x0;
    at = at0;
    while (true) {
      // a request: its units from cost `at` on
      r = l_scalar(r);
      x.q0 = l_scalar(x.q0);
      x.n = l_scalar(x.n);
      x.P = l_scalar(x.P);
      at = l_scalar(at);
      const int rows = x.rows(a), T = x.tiles();
      const int full_unit = whole ? 1 : l_unit_cost(T, 1 << us);
      int j = unit_of(x, at, from);
      at += j * full_unit;
      bool check = true, ok = true;
      for (; j << us < rows && at < to; ++j) {
        LatUnit u;
        u.w = wid;
        u.q0 = x.q0;
        u.n = x.n;
        u.P = x.P;
        u.r = r;
        u.row0 = l_scalar(j << us);
        u.rows = l_scalar(min(1 << us, rows - u.row0));
        u.tree_tiles = x.tree_tiles();
        const int c = l_tile_cost(u.rows);
        const int t_at = at + l_enter_cost(u.rows);  // where its tiles start
        const int t0 = l_scalar(whole ? 0 : l_tile_at(from - t_at, c, T));
        const int t1 = l_scalar(whole ? T : l_tile_at(to - t_at, c, T));
        if (ok && t0 < t1) {
          const size_t part = size_t(g) * 2 + (t0 == 0 ? 1 : 0);
          const bool all = t0 == 0 && t1 == T;
          ok = c == kLCost4           ? l_segment<2, false>(a, ws, u, t0, t1, all, part, check, base)
               : u.rows <= kLRestRows ? l_segment<1, true>(a, ws, u, t0, t1, all, part, check, base)
                                      : l_segment<1, false>(a, ws, u, t0, t1, all, part, check, base);
          check = false;
          if (!ok && tid == 0) status_or(a.status, ECHO_DATA_BAD_OFFSETS);
          // (the second of a unit's ranges has the record)
          if (ok && t0 > 0 && ranges.range_of(t_at) == g - 1 && tid == 0) {
            LatCut cut;
            cut.parts = ranges.range_of(t_at + (T - 1) * c) - g + 2;
            cut.rows = u.rows;
            cut.row = (long long)u.q0 * a.hq + u.row0;
            ws.cuts[g] = cut;
          }
        }
        at += whole ? 1 : l_unit_cost(T, u.rows);
      }
      if (at >= to) break;
      // the next request with rows
      int next = r + 1;
      for (; next < a.R; next += kWave) {
        x = LatLook{};
        if (next + lane < a.R) x = l_look(a, next + lane);
        const uint64_t in = __ballot(x.n > 0);
        if (in != 0ull) {
          const int i = __ffsll((unsigned long long)in) - 1;
          next += i;
          x.q0 = __shfl(x.q0, i);
          x.n = __shfl(x.n, i);
          x.P = __shfl(x.P, i);
          break;
        }
      }
      if (next >= a.R) break;
      r = next;
    }
  }
}

// ------------------------------------------------------------- combine ----

// Workgroup (g, y): of the unit in record g, rows 32 (y / 8) .. and dims 64 (y % 8) ..; a thread has
// eight dims of a row, in two pieces.  Parts in the order of the ranges.
__global__ __launch_bounds__(256) void latent_combine_kernel(LatArgs a, LatWs ws) {
  const int g = blockIdx.x;
  const const_i32_t* rec = (const const_i32_t*)(ws.cuts + g);  // (scalar loads)
  const int parts = rec[0], rows = rec[1];
  const int rt = int(blockIdx.y) / 8, rl = threadIdx.x & 31, row = 32 * rt + rl;
  if (parts == 0 || row >= rows) return;
  const int64_t first = int64_t(uint64_t(uint32_t(rec[2])) | (uint64_t(uint32_t(rec[3])) << 32));
  const int d4 = 16 * int(blockIdx.y & 7) + (threadIdx.x >> 5);
  float M = -__builtin_inff(), L = 0.0f, Lq = 0.0f;
  floatx4 acc[2] = {};
  for (int i0 = 0; i0 < parts; i0 += kLParts) {  // (a batch's loads in one round trip)
    floatx4 ml[kLParts], v[kLParts][2];
#pragma unroll
    for (int j = 0; j < kLParts; ++j) {
      ml[j] = floatx4{-__builtin_inff(), 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < 2; ++k) v[j][k] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
      if (i0 + j < parts) {  // uniform
        const size_t part = size_t(g - 1 + i0 + j) * 2 + (i0 + j == 0 ? 1 : 0);
        ml[j] = *reinterpret_cast<const floatx4*>(ws.part_ml + (part * kLRows + row) * 4);
        const float* po = ws.part_o + ((part * 4 + rt) * 128 + d4) * 128 + rl * 4;
#pragma unroll
        for (int k = 0; k < 2; ++k) v[j][k] = *reinterpret_cast<const floatx4*>(po + 8 * k * 128);
      }
    }
    float m = M;
#pragma unroll
    for (int j = 0; j < kLParts; ++j) m = fmaxf(m, ml[j][0]);
    if (m == -__builtin_inff()) continue;
    const float was = __builtin_amdgcn_exp2f(M - m);  // 0 from -inf
    M = m;
    L *= was;
    Lq *= was;
#pragma unroll
    for (int k = 0; k < 2; ++k) acc[k] *= was;
#pragma unroll
    for (int j = 0; j < kLParts; ++j) {
      const float w = __builtin_amdgcn_exp2f(ml[j][0] - m);  // 0 from -inf
      L = __builtin_fmaf(w, ml[j][1], L);
      Lq = __builtin_fmaf(w, ml[j][2], Lq);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[k][e] = __builtin_fmaf(w, v[j][k][e], acc[k][e]);
    }
  }
  const float inv = Lq > 0.0f ? 1.0f / Lq : 0.0f;
  uint16_t* out = a.out + (first + row) * kLC + 4 * d4;
#pragma unroll
  for (int k = 0; k < 2; ++k)
    *reinterpret_cast<uint2*>(out + 32 * k) =
        make_uint2(pack_bf16x2(acc[k][0] * inv, acc[k][1] * inv), pack_bf16x2(acc[k][2] * inv, acc[k][3] * inv));
  if (a.lse != nullptr && d4 == 0) a.lse[first + row] = L > 0.0f ? (M + log2f(L)) * kLn2 : -__builtin_inff();
}

}  // namespace

size_t attn_latent_workspace_bytes(int32_t R, int32_t max_pages) {
  size_t n = 0;
  l_layout(nullptr, R, max_pages, device_cu_count(), &n);
  return n;
}

int32_t launch_tree_verify_attn_latent(const AttnLatentArgs& x, hipStream_t stream) {
  (void)hipGetLastError();
  const int G = device_cu_count();
  const LatWs ws = l_layout(x.workspace, x.R, x.max_pages, G, nullptr);
  LatArgs a;
  a.q = x.q;
  a.latent_new = x.latent_new;
  a.pages = x.cache.pages;
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
  a.scale2 = x.sm_scale * kLog2e;
  a.out = x.out;
  a.lse = x.lse;
  a.status = x.status;
  a.chunks = l_page_chunks(a.max_pages);
  if (a.chunks > 0)
    hipLaunchKernelGGL(latent_pages_kernel, dim3(unsigned(a.chunks), unsigned(a.R)), dim3(kPageChunk), 0, stream, a,
                       ws.bad);
  hipLaunchKernelGGL(latent_main_kernel, dim3(unsigned(G)), dim3(kLThreads), 0, stream, a, ws);
  const long long rows = (long long)a.max_rows * a.hq;
  hipLaunchKernelGGL(latent_combine_kernel, dim3(unsigned(G), unsigned((rows < kLRows ? rows : kLRows) + 31) / 32 * 8),
                     dim3(256), 0, stream, a, ws);
  return hipGetLastError() == hipSuccess ? ECHO_OK : ECHO_ERR_HIP;
}

}  // namespace echo
