// The choice of the best candidates that a work-group's threads hold in registers: shared by the beam step and the label scores.
#pragma once
#include "common.h"

namespace lstm {
namespace {

constexpr int kBeamMax = 16;          // the most that are chosen

// (value, index) pairs ordered by larger value first, then smaller index: `better(a, b)` = a comes before b
struct Cand { float v; int i; };
__device__ __forceinline__ bool better(const Cand& a, const Cand& b) { return (a.v > b.v) | ((a.v == b.v) & (a.i < b.i)); }
// field by field: selecting between two structs made the compiler store both to scratch memory and load one back
__device__ __forceinline__ Cand pick(const Cand& a, const Cand& b) {
  const bool t = better(a, b);
  Cand c;
  c.v = t ? a.v : b.v;
  c.i = t ? a.i : b.i;
  return c;
}
// The best candidate of the wavefront, in every lane.  Six combining steps through DPP moves (neighbour in the quad, other
// pair of the quad, mirrored half row, mirrored row, last lane of the row before, last lane of the first half), after
// which lane 63 holds the result; 64 lanes of `__shfl_xor` took six dependent trips through the LDS crossbar per value.
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ Cand dpp_step(const Cand& c) {
  Cand d;   // lanes that the move does not reach (row mask, row_bcast sources out of range) keep their own candidate
  d.v = __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(c.v), __float_as_int(c.v), CTRL, ROW_MASK, 0xf, false));
  d.i = __builtin_amdgcn_update_dpp(c.i, c.i, CTRL, ROW_MASK, 0xf, false);
  return pick(c, d);
}
__device__ __forceinline__ Cand wave_best(Cand c) {
  c = dpp_step<0xB1, 0xf>(c);       // quad_perm [1,0,3,2]
  c = dpp_step<0x4E, 0xf>(c);       // quad_perm [2,3,0,1]
  c = dpp_step<0x141, 0xf>(c);      // row_half_mirror
  c = dpp_step<0x140, 0xf>(c);      // row_mirror: every lane holds the best of its row of 16
  c = dpp_step<0x142, 0xa>(c);      // row_bcast15 into rows 1 and 3
  c = dpp_step<0x143, 0xc>(c);      // row_bcast31 into rows 2 and 3
  Cand w;
  w.v = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(c.v), 63));
  w.i = __builtin_amdgcn_readlane(c.i, 63);
  return w;
}
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ unsigned dpp_max(unsigned c) { return max(c, (unsigned)__builtin_amdgcn_update_dpp((int)c, (int)c, CTRL, ROW_MASK, 0xf, false)); }
__device__ __forceinline__ unsigned wave_max(unsigned c) {        // (the same steps)
  c = dpp_max<0x142, 0xa>(dpp_max<0x140, 0xf>(dpp_max<0x141, 0xf>(dpp_max<0x4E, 0xf>(dpp_max<0xB1, 0xf>(c)))));
  return (unsigned)__builtin_amdgcn_readlane((int)dpp_max<0x143, 0xc>(c), 63);
}
// The choice of a work-group's best `need` candidates, best first, out of what its NW wavefronts hold in registers.
template <int NW>
struct Chooser {
  static constexpr int kSeg = NW == 1 ? 64 : 128;                // finalists a wavefront may contribute
  unsigned key[64 * NW];
  float v[NW][kSeg], out_v[kBeamMax], win_v[NW];
  int i[NW][kSeg], out_i[kBeamMax], win_i[NW], count[NW];
};
// `top` is the largest value this thread has seen (its own entries or earlier ones that the list so far holds), each(f) calls
// f(value, index) for every entry and scan(bound, f) for every entry that is not surely below the bound; both are wavefront-wide.  -inf and NaN are no candidates.  Results in s.out_v / out_i[0 .. need), (-inf, 0x7fffffff) where there are
// fewer; the caller synchronises before the next use of s.
// An entry strictly below the need-th largest of 64 values seen (a lane's `top`s, the largest of all wavefronts') has `need` entries in front of it.  That bound is found by bisection over
// the ordered bit patterns (20 bits of them, rounded down) between the least and the largest of the 64, a ballot a step, ended where exactly `need` are above (over 256 values with four ballots a step, and
// always 20 of them, it took 0.6 us more); what reaches it - little more than `need` entries unless values
// repeat - goes to a list in LDS, a stretch per wavefront, and the place of a finalist is the number of better ones.  Lists that do not
// fit (plateaus) are left: `need` rounds of "every thread offers its best behind the last winner" over the registers take their place.
template <int NW, typename Each, typename Scan>
__device__ __forceinline__ void choose_best(Chooser<NW>& s, float top, int need, Each each, Scan scan) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float kNegInf = -__builtin_inff();
  const unsigned f = __float_as_uint(top);
  unsigned key = ((f & 0x80000000u) ? ~f : (f | 0x80000000u)) >> 12;           // larger float => key not smaller
  if constexpr (NW > 1) {
    s.key[threadIdx.x] = key;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) key = max(key, s.key[64 * w + lane]);
  }
  constexpr unsigned kNone = 0x007fffffu >> 12;                   // the key of -inf: nothing seen
  float bound = kNegInf;
  if (__popcll(__ballot(key > kNone)) >= need) {
    unsigned hi = wave_max(key), lo = ~wave_max(key > kNone ? ~key : 0u);
    while (lo < hi) {
      const unsigned mid = lo + ((hi - lo) >> 1) + 1u;
      const int n = __popcll(__ballot(key >= mid));
      if (n >= need) lo = mid; else hi = mid - 1u;
      if (n == need) break;
    }
    const unsigned full = lo << 12;                               // the smallest ordered pattern with this key
    bound = __uint_as_float((full & 0x80000000u) ? (full & 0x7fffffffu) : ~full);
  }
  int count = 0;                                                 // of this wavefront (the same in every lane)
  scan(bound, [&](float x, int idx) {
    const bool keep = x > kNegInf && x >= bound;
    const unsigned long long mask = __ballot(keep);
    if (mask == 0ull) return;
    const int pos = count + (int)__popcll(mask & ((1ull << lane) - 1ull));
    if (keep && pos < Chooser<NW>::kSeg) { s.v[wave][pos] = x; s.i[wave][pos] = idx; }
    count += (int)__popcll(mask);
  });
  if (lane == 0) s.count[wave] = count;
  if (threadIdx.x < kBeamMax) { s.out_v[threadIdx.x] = kNegInf; s.out_i[threadIdx.x] = 0x7fffffff; }
  __syncthreads();
  int most = 0, total = 0, w = 0, at = threadIdx.x;                // thread t has finalist t of the stretches, number `at` of wavefront w's
#pragma unroll
  for (int q = 0; q < NW; ++q) {
    const int c = s.count[q];
    total += c;
    most = max(most, c);
    if (q + 1 < NW && (int)threadIdx.x >= total) { w = q + 1; at = threadIdx.x - total; }
  }
  if (most <= Chooser<NW>::kSeg && total <= 64 * NW) {
    const int t = threadIdx.x;
    if (wave * 64 >= total) return;
    Cand mine = {kNegInf, 0x7fffffff};
    if (t < total) { mine.v = s.v[w][at]; mine.i = s.i[w][at]; }
    int place = 0;
    if (NW == 1 || total <= 64) {
      for (int j = 0; j < total; ++j) {
        const Cand other = {__int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine.v), j)), __builtin_amdgcn_readlane(mine.i, j)};
        place += better(other, mine) ? 1 : 0;
      }
    } else {
#pragma unroll
      for (int seg = 0; seg < NW; ++seg) {
        const int n = s.count[seg];
        for (int j = 0; j < n; ++j) {
          const Cand other = {s.v[seg][j], s.i[seg][j]};
          place += better(other, mine) ? 1 : 0;
        }
      }
    }
    if (t < total && place < need) { s.out_v[place] = mine.v; s.out_i[place] = mine.i; }
    return;
  }
  Cand last = {__builtin_inff(), -1};                             // in front of every candidate
  for (int k = 0; k < need; ++k) {
    Cand mine = {kNegInf, 0x7fffffff};
    each([&](float x, int idx) {                                 // (-inf is sorted out below: a test of x alone would be kept for all rounds, in registers)
      const Cand c = {x, idx};
      if (better(last, c) && better(c, mine)) { mine.v = x; mine.i = idx; }
    });
    const Cand win = wave_best(mine);
    Cand best = win;
    if constexpr (NW > 1) {
      if (lane == 0) { s.win_v[wave] = win.v; s.win_i[wave] = win.i; }
      __syncthreads();
#pragma unroll
      for (int q = 0; q < NW; ++q) best = pick(best, Cand{s.win_v[q], s.win_i[q]});
    }
    if (threadIdx.x == 0 && best.v > kNegInf) { s.out_v[k] = best.v; s.out_i[k] = best.i; }
    last = best;
    __syncthreads();
  }
}

// What exponentials are taken relative to where the maximum may be -inf (nothing but -inf and NaN so far): exp(-inf - base) is 0 then, and a NaN stays one.
__device__ __forceinline__ float lse_base(float m) { return fmaxf(m, -__FLT_MAX__); }

}  // namespace
}  // namespace lstm
