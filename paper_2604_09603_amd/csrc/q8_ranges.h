// How the steps of the 8-bit attention are cut into ranges (attn_q8.hip says what units,
// steps, gangs and classes are): arithmetic on whole numbers alone, which the kernel and the
// host's tests share.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define ECHO_RANGES_UNROLL _Pragma("unroll")
#define ECHO_RANGES_FN __host__ __device__ __forceinline__
#else
#define ECHO_RANGES_UNROLL
#define ECHO_RANGES_FN inline
#endif

namespace echo {
namespace {

constexpr int kQ8Rows = 32;      // rows per unit
constexpr int kQ8Waves = 4;      // waves per workgroup
constexpr int kQ8StepKeys = 64;  // keys per step of the main loop: two tiles
constexpr int kQ8TreeKeys = 32;  // keys per step of the tree
constexpr int kQ8Classes = 3;    // gangs of k = 1 << class waves

ECHO_RANGES_FN int smaller(int a, int b) { return a < b ? a : b; }
ECHO_RANGES_FN int larger(int a, int b) { return a < b ? b : a; }

// What a step costs a workgroup that has 4, 2 or 1 gangs at work, relative to each other: between
// the ratios of their products (1, 2, 4) and those of their copies (4 : 2 : 1 gangs, so 1, 1, 1).
// 235B-shaped trees of 1 to 12 slots: 1, 2, 4 took 8 us more, 1, 1.5, 2.5 took 2 us more.
constexpr float kQ8Cost1 = 1.4f, kQ8Cost2 = 2.2f, kQ8Cost4 = 3.6f;
// Entering a unit (its rows of Q, the way out of the last one) takes as long as this many steps.
constexpr int kQ8Enter = 1;
// Of 32 steps that two gangs on the same CU share, the older workgroup's gets this many (17 in a
// class of gangs of four, which are bound by their products): its loads and products go
// first.  With these shares both end their ranges within a few us of each other.
constexpr int kQ8Older = 18;
constexpr float kQ8MaxSteps = 1073741824.0f;  // 2^30: steps of a call

// Workgroups b and b + half the grid share a CU (no result depends on it): places 2 b and
// 2 b + 1, so that a class has as many of the older as of the younger.
ECHO_RANGES_FN int q8_place(int b, int wgs) {
  return b < wgs / 2 ? 2 * b : 2 * (b - wgs / 2) + 1;
}
ECHO_RANGES_FN int q8_first_wave(int place, int wgs) {
  return ((place & 1) * (wgs / 2) + (place >> 1)) * kQ8Waves;
}

// How often class c goes through the keys of a head with t tiles of 32 rows.
ECHO_RANGES_FN int q8_passes(int t, int c) {
  const int rest = t & 3;
  return c == 2 ? (t >> 2) + (rest == 3 ? 1 : 0) : rest == c + 1 ? 1 : 0;
}

ECHO_RANGES_FN int q8_row_tiles(int nslots, int G) {
  return int((unsigned(nslots) * unsigned(G) + kQ8Rows - 1) / kQ8Rows);
}

// Steps of a unit: those of entering it (nothing is done in them), the tree's, the prefix's.
ECHO_RANGES_FN int q8_unit_steps(int nslots, int P) {
  return kQ8Enter + (nslots + kQ8TreeKeys - 1) / kQ8TreeKeys +
         int((unsigned(P) + kQ8StepKeys - 1) / kQ8StepKeys);
}

// T > 0 steps in ranges, of which two make a pair (one of its own if T = 1): pairs of equal
// size but for one step, and the first of two has older / 32 of the pair's steps.
// No range before the last is empty.
struct Q8Cutter {
  int n, each, more, older;
  ECHO_RANGES_FN Q8Cutter(int T, int gangs, int older_)
      : n(larger(smaller(gangs, T) / 2, 1)), older(older_) {
    each = int(unsigned(T) / unsigned(n));
    more = T - each * n;
  }
  ECHO_RANGES_FN int pair_at(int p) const { return p * each + smaller(p, more); }
  ECHO_RANGES_FN int first(int g) const {
    const int p = g >> 1, lo = pair_at(p);
    if ((g & 1) == 0) return lo;
    const int len = each + (p < more ? 1 : 0);
    return lo + smaller((len * older + 16) / 32, larger(len - 1, 1));
  }
  ECHO_RANGES_FN int range_of(int t) const {
    const int longer = more * (each + 1);
    const int p = t < longer ? int(unsigned(t) / unsigned(each + 1))
                             : more + int(unsigned(t - longer) / unsigned(each));
    return 2 * p + (t >= first(2 * p + 1) ? 1 : 0);
  }
};

// The steps of a call.  Offsets that overlap, or prefixes of shared pages, may ask for any number
// of them: the counts wrap then, the float tells.
struct Q8Steps {
  uint32_t of[kQ8Classes] = {0u, 0u, 0u};
  float all = 0.0f;
  ECHO_RANGES_FN void add(int hkv, int tiles, int tpu) {  // a request with tiles > 0
    const uint32_t pass = uint32_t(hkv) * uint32_t(tpu);
ECHO_RANGES_UNROLL
    for (int c = 0; c < kQ8Classes; ++c) {
      const int n = q8_passes(tiles, c);
      of[c] += pass * uint32_t(n);
      all += float(hkv) * float(tpu) * float(n);
    }
  }
};

// Whether a call asks for more steps than it may; then it has none.
ECHO_RANGES_FN bool q8_refuses(float all, int (&tot)[kQ8Classes]) {
  const bool no = !(all <= kQ8MaxSteps);
ECHO_RANGES_UNROLL
  for (int c = 0; c < kQ8Classes; ++c) tot[c] = no ? 0 : tot[c];
  return no;
}

// The workgroups at places wg0 .. wg0 + nwg - 1 take class cls.
struct Q8Share {
  int cls, wg0, nwg;
};

// What place g of wgs takes of a call with tot[c] >= 0 steps of class c: places go to the classes in
// pairs, by cost, at least one pair where there is work (per: places per cost of all of it).
ECHO_RANGES_FN float q8_cost(const int (&tot)[kQ8Classes], int c) {
  return (c == 0 ? kQ8Cost1 : c == 1 ? kQ8Cost2 : kQ8Cost4) * float(tot[c]);
}
ECHO_RANGES_FN Q8Share q8_share(const int (&tot)[kQ8Classes], int wgs, float per, int g) {
  Q8Share x = {0, 0, 0};
  int left = wgs, need = 0;
ECHO_RANGES_UNROLL
  for (int c = 0; c < kQ8Classes; ++c) need += tot[c] > 0 ? 1 : 0;
ECHO_RANGES_UNROLL
  for (int c = 0; c < kQ8Classes; ++c) {
    int n = 0;
    if (tot[c] > 0) {
      need -= 1;
      n = need == 0 ? left
                    : smaller(larger(2 * int(0.5f * per * q8_cost(tot, c) + 0.5f), 2), left - 2 * need);
    }
    if (g >= wgs - left && g < wgs - left + n) x = Q8Share{c, wgs - left, n};
    left -= n;
  }
  return x;
}

// Steps [lo, hi) of class 0, 1, 2 (gangs of k = 1, 2, 4 waves), which gang number `gang` of it takes.
struct Q8Range {
  Q8Cutter ranges;  // of the class
  int lo, hi, k, member, gang, wg0, nwg;
};

// The range of wave wid of the workgroup at place g, whose class has `steps` steps.  None where
// there are none; x has no places then.
ECHO_RANGES_FN Q8Range q8_range_at(const Q8Share& x, int steps, int g, int wid) {
  Q8Range r = {Q8Cutter(larger(steps, 1), x.nwg * (kQ8Waves >> x.cls), kQ8Older - (x.cls == 2 ? 1 : 0)),
               0, 0, 1 << x.cls, wid & ((1 << x.cls) - 1), g - x.wg0 + (wid >> x.cls) * x.nwg, x.wg0,
               x.nwg};
  if (steps > 0 && r.gang < 2 * r.ranges.n) {
    r.lo = r.ranges.first(r.gang);
    r.hi = r.ranges.first(r.gang + 1);
  }
  return r;
}

}  // namespace
}  // namespace echo
