// Log probabilities of given labels under the softmax of an output layer's logits, with entropy, best alternatives and gradient:
//
//     m = max x,  z = sum e^(x - m)      logp = (x[label] - m) - log z      entropy = log z - (sum e^(x - m) (x - m)) / z
//     dlogits[v] = dlogp ([v = label] - p[v]) - dent p[v] (log p[v] + entropy),  log p = (x - m) - log z
//
// m, z and u = sum e^(x - m) (x - m) are kept running: where m grows by d, z' = z e^-d and u' = (u - d z) e^-d.
#include <algorithm>
#include <type_traits>

#include "../../include/lstm_abi.h"
#include "choose_dev.h"
#include "common.h"
#include "exchange_dev.h"

#pragma clang fp contract(off)        // products and sums are fused where it says fma; the forms of a kernel differ in the order of their sums alone

namespace lstm {
namespace {

constexpr int kTopMax = kBeamMax;
constexpr int kVocabMost = 1 << 26;
constexpr int kPieces = 24;           // 16-byte pieces of a row that a thread holds at most where they are kept
constexpr int kStretches = 32;        // stretches of a row at most
constexpr long kStretchGroups = 768;  // work-groups up to which rows are cut into stretches
constexpr long kWholeRows = 256;      // rows, and labels of a row, whose alternatives sixteen wavefronts choose in one launch
constexpr int kWholeFrom = 4096, kWholeTo = 32768;

typedef __attribute__((ext_vector_type(2))) float f32x2_;
typedef __attribute__((ext_vector_type(2))) bf16_t bf16x2_;

struct ScoreArgs {
  const void* x; long ld;
  const int* label; const int* lens;
  float* logp; float* entropy; float2* stats;
  float* top_logp; int* top_label;
  const float2* stats_in; const float* entropy_in; const float* dlogp; const float* dent;
  void* dx; long ldd;
  float4* sums; float* cand_val; int* cand_lab;         // of the stretches: [row][parts], [row][parts][top]
  int T, B, V, top;
  int parts, per, step;                                 // stretches of a row, pieces of a stretch, pieces of a round
};
__device__ __forceinline__ bool padded(const ScoreArgs& a, int r) { return a.lens && r / a.B >= a.lens[r % a.B]; }

// A row between its first and its last 16-byte boundary, in pieces of E values, and the up to 2 (E - 1) values outside them.
template <typename T> struct Pieces;
template <> struct Pieces<float> {
  static constexpr int E = 4;
  static __device__ __forceinline__ float get(const u32x4& w, int e) { return __uint_as_float(w[e]); }
};
template <> struct Pieces<bf16_t> {
  static constexpr int E = 8;
  static __device__ __forceinline__ float get(const u32x4& w, int e) { return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16); }
};
template <typename T> struct RowOf {
  static constexpr int E = Pieces<T>::E;
  int head, pieces, tail;
  __device__ __forceinline__ RowOf(const T* row, int V) {
    head = min(V, (int)((-(uintptr_t)row & 15) / sizeof(T)));
    pieces = (V - head) / E;
    tail = V - head - pieces * E;
  }
  __device__ __forceinline__ int outside(int i) const { return i < head ? i : head + pieces * E + i - head; }      // the i-th value outside the pieces
};

// What a row's exponentials add up to relative to m: z = sum e^(x - m), u = sum e^(x - m) (x - m) / ln 2; -inf, 0, 0 is the empty sum.  A value that is
// far below takes part as 2^-20000 of itself, 0, and so does -inf, without a product of 0 and infinity.
struct Sums { float m, z, u; };
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f, kFar = -20000.f;
__device__ __forceinline__ float base_of(float m) { return fmaxf(m, -__FLT_MAX__); }    // (no -inf - -inf)
__device__ __forceinline__ void move_base(Sums& s, float m) {
  const float d = fmaxf((base_of(s.m) - base_of(m)) * kLog2e, kFar), e = __builtin_amdgcn_exp2f(d);
  s.u = fmaf(d, s.z, s.u) * e;
  s.z *= e;
  s.m = m;
}
__device__ __forceinline__ void add(Sums& s, float base, float x) {                     // base = base_of(s.m); NaN and +inf make z and u NaN
  const float t = (x - base) * kLog2e, e = __builtin_amdgcn_exp2f(t);
  s.z += e;
  s.u = fmaf(e, fmaxf(t, kFar), s.u);
}
__device__ __forceinline__ Sums join(Sums a, Sums b) {
  const float m = fmaxf(a.m, b.m);
  move_base(a, m);
  move_base(b, m);
  return {m, a.z + b.z, a.u + b.u};
}
template <int NW>
__device__ __forceinline__ Sums join_all(Sums s, Sums* part) {                          // over a work-group of NW wavefronts, in every thread
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const Sums other = {__shfl_xor(s.m, o), __shfl_xor(s.z, o), __shfl_xor(s.u, o)};
    s = join(s, other);
  }
  if constexpr (NW > 1) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    s = part[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) s = join(s, part[w]);
  }
  return s;
}
template <typename T>
__device__ __forceinline__ void write_values(const ScoreArgs& a, int r, const T* row, const Sums& s, float logz) {      // by one thread
  const bool pad = padded(a, r), empty = s.z == 0.f;
  const float m = s.z != s.z ? s.z : s.m;                        // (a row of NaN has no maximum, and is not an empty one)
  if (a.stats) a.stats[r] = pad ? make_float2(0.f, 0.f) : empty ? make_float2(-__builtin_inff(), 0.f) : make_float2(m, logz);
  if (a.entropy) a.entropy[r] = pad || empty ? 0.f : logz - kLn2 * (s.u / s.z);
  if (a.logp) {
    const int l = a.label[r];
    float p = 0.f;
    if (!pad && l >= 0 && l < a.V) p = empty ? -__builtin_inff() : (Store<T>::load(row, l) - s.m) - logz;
    a.logp[r] = p;
  }
}

// Row r in a.parts stretches, a work-group each (several for few rows, which would leave compute units idle).  A stretch is read once, up to U loads of
// 16 bytes a thread in flight, and folded a few pieces at a time (two without alternatives, which
// leaves little of the last round empty: 3200 rows of 20000 bfloat16 values 48 us with four, 36 with two); where alternatives are wanted it stays in registers and they are chosen there as in the beam
// step: one bound for the whole work-group tells the few entries that can be among the best apart, and these are ranked.  A stretch of more than 64 NW U pieces
// takes several rounds, each with the best so far among its candidates.  2048 rows of 131071 float values 182 us (5.9 TB/s, memory); 3200 of 20000 bfloat16 ones 36 to 47
// (the exponentials: two a value); 768 of 20000 float with 5 alternatives 15 (all rows at once: loads, then choices).
template <typename T, bool TOP, int U, int NW, bool STREAM = false>
__global__ __launch_bounds__(64 * NW) void label_score_kernel(ScoreArgs a) {
  typedef Pieces<T> P;
  constexpr int NT = 64 * NW, E = P::E, G = U < 2 ? U : TOP && U % 4 == 0 ? 4 : 2;
  static_assert(U % G == 0, "pieces are folded G at a time");
  __shared__ Sums part[NW];
  __shared__ typename std::conditional<TOP, Chooser<NW>, int>::type s;
  const int r = (int)blockIdx.x / a.parts, stretch = (int)blockIdx.x - r * a.parts, tid = threadIdx.x;
  const float kNegInf = -__builtin_inff();
  const T* row = (const T*)a.x + (long)r * a.ld;
  const RowOf<T> at(row, a.V);
  const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)(row + at.head), 0, at.pieces * 16, kBufFlags);
  if (padded(a, r)) {                 // nothing of it is read (with several stretches the merge writes its values)
    if (a.parts == 1) {
      if (tid == 0) write_values(a, r, row, {kNegInf, 0.f, 0.f}, 0.f);
      if (TOP && tid < a.top) { a.top_logp[(long)r * a.top + tid] = kNegInf; a.top_label[(long)r * a.top + tid] = 0; }
    }
    return;
  }
  const int begin = stretch * a.per, end = min(at.pieces, begin + a.per);
  Sums sum = {kNegInf, 0.f, 0.f};
  float ex = kNegInf;                 // an entry outside the pieces: first the row's own, later one of the best so far
  int ei = 0x7fffffff;
  if (stretch == 0 && tid < at.head + at.tail) {
    ei = at.outside(tid);
    ex = Store<T>::load(row, ei);
    sum.m = fmaxf(ex, kNegInf);
    add(sum, base_of(sum.m), ex);
  }
  float top = sum.m;
  for (int base = begin;; ) {
    const int stop = min(end, base + a.step);
    u32x4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = __builtin_amdgcn_raw_buffer_load_b128(rs, (unsigned)(base + u * NT + tid) * 16u, 0, STREAM ? 2 : 0);      // (2: non-temporal)
    if (base + U * NT > stop) {       // pieces behind the end hold -inf
      const int left = stop - base - tid;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < 4; ++q) w[u][q] = u * NT < left ? w[u][q] : sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
    }
#pragma unroll
    for (int u0 = 0; u0 < U; u0 += G) {
      if (!TOP && base + u0 * NT >= stop) break;
      float m = sum.m;
#pragma unroll
      for (int u = u0; u < u0 + G; ++u)
#pragma unroll
        for (int e = 0; e < E; ++e) m = fmaxf(m, P::get(w[u], e));
      move_base(sum, m);
      const float b = base_of(m);
#pragma unroll
      for (int u = u0; u < u0 + G; ++u)
#pragma unroll
        for (int e = 0; e < E; ++e) add(sum, b, P::get(w[u], e));
    }
    if constexpr (TOP) {
      const int first = at.head + E * (base + tid);
      const auto each = [&](auto f) {
        int i = first;
        asm volatile("" : "+v"(i));                              // (or all labels are kept in registers for the rounds behind a full list)
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < E; ++e) f(P::get(w[u], e), i + E * NT * u + e);
        f(ex, ei);
      };
      const auto scan = [&](float bound, auto f) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float most = P::get(w[u], 0);
#pragma unroll
          for (int e = 1; e < E; ++e) most = fmaxf(most, P::get(w[u], e));
          if (__ballot(most >= bound) == 0ull) continue;
#pragma unroll
          for (int e = 0; e < E; ++e) f(P::get(w[u], e), first + E * NT * u + e);
        }
        f(ex, ei);
      };
      top = sum.m;
      choose_best(s, top, a.top, each, scan);
    }
    base += a.step;
    if (base >= end) break;
    if constexpr (TOP) {
      __syncthreads();
      ex = tid < a.top ? s.out_v[tid] : kNegInf;
      ei = tid < a.top ? s.out_i[tid] : 0x7fffffff;
      __syncthreads();
    }
  }
  sum = join_all<NW>(sum, part);
  if (a.parts > 1) {
    if (tid == 0) a.sums[blockIdx.x] = make_float4(sum.m, sum.z, sum.u, 0.f);
    if constexpr (TOP) {
      __syncthreads();
      if (tid < a.top) {
        a.cand_val[(long)blockIdx.x * a.top + tid] = s.out_v[tid];
        a.cand_lab[(long)blockIdx.x * a.top + tid] = s.out_i[tid];
      }
    }
    return;
  }
  const float logz = logf(sum.z);
  if (tid == 0) write_values(a, r, row, sum, logz);
  if constexpr (TOP) {
    __syncthreads();
    if (tid < a.top) {
      const bool found = s.out_i[tid] != 0x7fffffff && logz - logz == 0.f;       // (a NaN among the row's logits: none)
      a.top_logp[(long)r * a.top + tid] = found ? (s.out_v[tid] - sum.m) - logz : kNegInf;
      a.top_label[(long)r * a.top + tid] = found ? s.out_i[tid] : 0;
    }
  }
}

// The stretches of row r = blockIdx.x: their sums, and the best of their best.  One wavefront.
template <typename T, int N>
__global__ __launch_bounds__(64) void label_score_merge_kernel(ScoreArgs a) {
  __shared__ Chooser<1> s;
  const int r = blockIdx.x, tid = threadIdx.x, total = a.parts * a.top;
  const float kNegInf = -__builtin_inff();
  if (padded(a, r)) {
    if (tid == 0) write_values(a, r, (const T*)a.x + (long)r * a.ld, {kNegInf, 0.f, 0.f}, 0.f);
    if (tid < a.top) { a.top_logp[(long)r * a.top + tid] = kNegInf; a.top_label[(long)r * a.top + tid] = 0; }
    return;
  }
  Sums sum = {kNegInf, 0.f, 0.f};
  float v[N];
  int i[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int c = tid + 64 * k;
    v[k] = c < total ? a.cand_val[(long)r * total + c] : kNegInf;
    i[k] = c < total ? a.cand_lab[(long)r * total + c] : 0x7fffffff;
  }
  if (tid < a.parts) {
    const float4 p = a.sums[(long)r * a.parts + tid];
    sum = {p.x, p.y, p.z};
  }
  sum = join_all<1>(sum, nullptr);
  const float logz = logf(sum.z);
  if (tid == 0) write_values(a, r, (const T*)a.x + (long)r * a.ld, sum, logz);
  if (a.top == 0) return;
  float top = kNegInf;
#pragma unroll
  for (int k = 0; k < N; ++k) top = fmaxf(top, v[k]);
  const auto each = [&](auto f) {
#pragma unroll
    for (int k = 0; k < N; ++k) f(v[k], i[k]);
  };
  choose_best(s, top, a.top, each, [&](float, auto f) { each(f); });
  __syncthreads();
  if (tid < a.top) {
    const bool found = s.out_i[tid] != 0x7fffffff && logz - logz == 0.f;
    a.top_logp[(long)r * a.top + tid] = found ? (s.out_v[tid] - sum.m) - logz : kNegInf;
    a.top_label[(long)r * a.top + tid] = found ? s.out_i[tid] : 0;
  }
}

// dlogits: a work-group takes up to kBwdPieces pieces a thread of one row, read and written once (2048 rows of 131071 float values 379 us, 5.7 TB/s: memory).  Rows of logits and of dlogits that lie differently to the
// 16-byte boundaries go value by value.
constexpr int kBwdPieces = 4;
template <typename T, bool STREAM>
__global__ __launch_bounds__(256) void label_score_bwd_kernel(ScoreArgs a) {
  typedef Pieces<T> P;
  constexpr int E = P::E;
  const int r = (int)blockIdx.x / a.parts, stretch = (int)blockIdx.x - r * a.parts, tid = threadIdx.x;
  const T* row = (const T*)a.x + (long)r * a.ld;
  T* out = (T*)a.dx + (long)r * a.ldd;
  const bool pad = padded(a, r);
  int l = a.dlogp && !pad ? a.label[r] : -1;
  if (l < 0 || l >= a.V) l = -1;
  const float dl = l >= 0 ? a.dlogp[r] : 0.f, de = a.dent && !pad ? a.dent[r] : 0.f, h = a.dent && !pad ? a.entropy_in[r] : 0.f;
  const float2 st = pad ? make_float2(0.f, 0.f) : a.stats_in[r];
  const bool none = pad || (dl == 0.f && de == 0.f) || st.x == -__builtin_inff(), plain = de == 0.f;
  const auto value = [&](float x, int v) {
    const float q = (x - st.x) - st.y, p = __builtin_amdgcn_exp2f(q * kLog2e);
    return fmaf(-p, plain ? dl : fmaf(de, fmaxf(q, kFar) + h, dl), v == l ? dl : 0.f);
  };
  const RowOf<T> at(row, a.V);
  if (((uintptr_t)row ^ (uintptr_t)out) & 15) {
    const int begin = stretch * 256 * kBwdPieces * E, end = stretch + 1 == a.parts ? a.V : min(a.V, begin + 256 * kBwdPieces * E);
    for (int v = begin + tid; v < end; v += 256) Store<T>::store(out, v, none ? 0.f : value(Store<T>::load(row, v), v));
    return;
  }
  const u32x4* from = (const u32x4*)(row + at.head);
  u32x4* to = (u32x4*)(out + at.head);
  const int begin = stretch * 256 * kBwdPieces;
  u32x4 w[kBwdPieces];
#pragma unroll
  for (int u = 0; u < kBwdPieces; ++u) {
    const int p = begin + u * 256 + tid;
    w[u] = u32x4{0u, 0u, 0u, 0u};
    if (!none && p < at.pieces) w[u] = STREAM ? __builtin_nontemporal_load(from + p) : from[p];
  }
  if (stretch == 0 && tid < at.head + at.tail) {
    const int v = at.outside(tid);
    Store<T>::store(out, v, none ? 0.f : value(Store<T>::load(row, v), v));
  }
#pragma unroll
  for (int u = 0; u < kBwdPieces; ++u) {
    const int p = begin + u * 256 + tid, v0 = at.head + p * E;
    if (p >= at.pieces) break;
    if (!none) {
      float d[E];
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] = value(P::get(w[u], e), v0 + e);
      if constexpr (E == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[u][e] = __float_as_uint(d[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x2_ x = {d[2 * e], d[2 * e + 1]};
          w[u][e] = __builtin_bit_cast(unsigned, __builtin_convertvector(x, bf16x2_));
        }
      }
    }
    if (STREAM) __builtin_nontemporal_store(w[u], to + p); else to[p] = w[u];
  }
}

int score_dims(int T, int B, int V, int top) {
  if (T < 0 || B < 0 || V < 1 || top < 0 || (long)T * B >= 1L << 23) return LSTM_ERR_DIM;
  if (V > kVocabMost || top > kTopMax) return LSTM_ERR_UNSUPPORTED;
  return LSTM_OK;
}
// Alternatives of few rows that sixteen wavefronts hold at once, a row a compute unit: one launch instead of stretches and their merge (8 alternatives, us in a replayed
// graph: 1 row of 5000 float 7.3 against 8.3, 1 of 20000 8.6 both, 100 of 20000 9.4 against 11.3, and 3 us less on
// the host; 400 rows, two a compute unit, 19.8 against 12.3). Scores alone
// are read faster than the wider meeting ends (1 row of 20000 6.1 against 5.2).
bool whole_rows(long rows, int V, int top) { return top > 0 && rows <= kWholeRows && V > kWholeFrom && V <= kWholeTo; }
// Stretches a row is cut into: as many as the device holds at once (three work-groups a compute unit), of at least 2048 entries.
int stretches(long rows, int V, int top) { return rows < 1 || whole_rows(rows, V, top) ? 1 : (int)std::max(1L, std::min({(long)kStretches, kStretchGroups / rows, (long)V / 2048})); }
uint64_t whole(uint64_t b) { return (b + 255) / 256 * 256; }
uint64_t score_bytes(long rows, int parts, int top) {
  return parts == 1 ? 0 : 256 + whole((uint64_t)rows * parts * sizeof(float4)) + 2 * whole((uint64_t)rows * parts * top * 4);
}
// Logits that the last-level cache does not hold (us: 2048 rows of 131071 float 204 -> 198 forward, 383 -> 372 backward; 5120 of 20000 152 -> 131 backward; 64 of 131071,
// which fit, 12 -> 15).
template <typename T> bool streams(const ScoreArgs& a) { return (uint64_t)a.T * a.B * a.V * sizeof(T) > kLastLevelBytes; }
template <typename T, bool TOP>
void launch_rows(ScoreArgs a, hipStream_t s) {
  if constexpr (!TOP) {
    // Many short rows: a wavefront each, nothing to meet over (4000 rows of 1000 bfloat16 values 11.7 us a call with four, 8.3 with one); few of them
    // would leave each compute unit a wavefront or two.
    if (a.parts == 1 && a.step > 64 && a.step <= 512 && (long)a.T * a.B >= 2048) {
      const auto kernel = a.step <= 128 ? label_score_kernel<T, false, 2, 1> : a.step <= 256 ? label_score_kernel<T, false, 4, 1> : label_score_kernel<T, false, 8, 1>;
      hipLaunchKernelGGL(kernel, dim3((unsigned)(a.T * a.B)), dim3(64), 0, s, a);
      return;
    }
  }
  if constexpr (TOP) {
    if (whole_rows((long)a.T * a.B, a.V, a.top)) {
      a.step = a.per;                                           // (one round: at most 8 pieces a thread of float, 4 of bfloat16)
      const int w = cdiv(a.per, 1024);
      auto kernel = w <= 2 ? label_score_kernel<T, true, 2, 16> : label_score_kernel<T, true, 4, 16>;
      if constexpr (Pieces<T>::E == 4) kernel = w <= 4 ? kernel : w <= 6 ? label_score_kernel<T, true, 6, 16> : label_score_kernel<T, true, 8, 16>;
      hipLaunchKernelGGL(kernel, dim3((unsigned)(a.T * a.B)), dim3(1024), 0, s, a);
      return;
    }
  }
  const int u = cdiv(a.step, 256);
  const auto row = [&](auto kernel, int waves) { hipLaunchKernelGGL(kernel, dim3((unsigned)(a.T * a.B * a.parts)), dim3(64 * waves), 0, s, a); };
  if (a.step <= 64) row(label_score_kernel<T, TOP, 1, 1>, 1);
  else if (u <= 1) row(label_score_kernel<T, TOP, 1, 4>, 4);
  else if (u <= 2) row(label_score_kernel<T, TOP, 2, 4>, 4);
  else if (u <= 4) row(label_score_kernel<T, TOP, 4, 4>, 4);
  else if (u <= 8) row(label_score_kernel<T, TOP, 8, 4>, 4);
  else if (u <= 12) row(label_score_kernel<T, TOP, 12, 4>, 4);
  else if (!TOP && streams<T>(a)) row(label_score_kernel<T, false, 16, 4, true>, 4);
  else if (!TOP || u <= 16) row(label_score_kernel<T, TOP, 16, 4>, 4);
  else if constexpr (TOP) row(u <= 20 ? label_score_kernel<T, TOP, 20, 4> : label_score_kernel<T, TOP, kPieces, 4>, 4);
}
template <typename T>
void launch_score(ScoreArgs a, hipStream_t s) {
  constexpr int E = Pieces<T>::E;
  a.per = cdiv(cdiv(a.V, E), a.parts);
  a.step = cdiv(a.per, cdiv(a.per, 256 * (a.top > 0 ? kPieces : 16)));            // pieces of a round: rounds of one length
  if (a.top > 0) launch_rows<T, true>(a, s); else launch_rows<T, false>(a, s);
  if (a.parts == 1) return;
  const int c = a.parts * a.top;
  const auto merge = c <= 64 ? label_score_merge_kernel<T, 1> : c <= 256 ? label_score_merge_kernel<T, 4> : label_score_merge_kernel<T, kStretches * kTopMax / 64>;
  hipLaunchKernelGGL(merge, dim3((unsigned)(a.T * a.B)), dim3(64), 0, s, a);
}

}  // namespace
}  // namespace lstm

using namespace lstm;

extern "C" {

int lstm_label_score_query(int T, int B, int V, int top, uint64_t* workspace_bytes) {
  if (!workspace_bytes) return LSTM_ERR_NULL;
  const int rc = score_dims(T, B, V, top);
  if (rc) return rc;
  *workspace_bytes = score_bytes((long)T * B, stretches((long)T * B, V, top), top);
  return LSTM_OK;
}

int lstm_label_score_fwd(int dtype, int T, int B, int V, const void* logits, int64_t ld, const int32_t* label, const int32_t* seq_lens,
                         float* logp, float* entropy, float* stats, int top, float* top_logp, int32_t* top_label, void* workspace,
                         uint64_t workspace_bytes, void* stream) {
  const bool any = T > 0 && B > 0;                             // (arrays without elements may have no address)
  if (any && (!logits || (logp && !label) || (top > 0 && (!top_logp || !top_label)))) return LSTM_ERR_NULL;
  int rc = score_dims(T, B, V, top);
  if (rc) return rc;
  if (ld < V) return LSTM_ERR_DIM;
  if (dtype != LSTM_F32 && dtype != LSTM_BF16_F32STATE) return LSTM_ERR_UNSUPPORTED;
  if (((uintptr_t)logits & (dtype == LSTM_F32 ? 3 : 1)) || (((uintptr_t)label | (uintptr_t)seq_lens | (uintptr_t)logp | (uintptr_t)entropy |
      (uintptr_t)top_logp | (uintptr_t)top_label) & 3) || ((uintptr_t)stats & 7))
    return LSTM_ERR_ALIGN;
  const int parts = stretches((long)T * B, V, top);
  const uint64_t need = score_bytes((long)T * B, parts, top);
  if (need > 0 && !workspace) return LSTM_ERR_NULL;
  if (workspace_bytes < need) return LSTM_ERR_SIZE;
  if (T == 0 || B == 0) return LSTM_OK;
  if ((rc = device_ok())) return rc;
  ScoreArgs a = {};
  a.x = logits; a.ld = ld; a.label = label; a.lens = seq_lens; a.logp = logp; a.entropy = entropy; a.stats = (float2*)stats; a.top = top; a.top_logp = top_logp;
  a.top_label = top_label; a.T = T; a.B = B; a.V = V; a.parts = parts;
  char* ws = (char*)(((uintptr_t)workspace + 255) / 256 * 256);
  a.sums = (float4*)ws;
  a.cand_val = (float*)(ws + whole((uint64_t)T * B * parts * sizeof(float4)));
  a.cand_lab = (int*)((char*)a.cand_val + whole((uint64_t)T * B * parts * top * 4));
  if (dtype == LSTM_F32) launch_score<float>(a, (hipStream_t)stream); else launch_score<bf16_t>(a, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? LSTM_OK : LSTM_ERR_HIP;
}

int lstm_label_score_bwd(int dtype, int T, int B, int V, const void* logits, int64_t ld, const int32_t* label, const int32_t* seq_lens,
                         const float* stats, const float* entropy, const float* dlogp, const float* dent, void* dlogits, int64_t ldd, void* stream) {
  if (T > 0 && B > 0 && (!logits || !stats || !dlogits || (dlogp && !label) || (dent && !entropy))) return LSTM_ERR_NULL;
  int rc = score_dims(T, B, V, 0);
  if (rc) return rc;
  if (ld < V || ldd < V) return LSTM_ERR_DIM;
  if ((dtype != LSTM_F32 && dtype != LSTM_BF16_F32STATE) || (dlogits == logits && ldd != ld)) return LSTM_ERR_UNSUPPORTED;
  if ((((uintptr_t)logits | (uintptr_t)dlogits) & (dtype == LSTM_F32 ? 3 : 1)) || (((uintptr_t)label | (uintptr_t)seq_lens |
      (uintptr_t)entropy | (uintptr_t)dlogp | (uintptr_t)dent) & 3) || ((uintptr_t)stats & 7))
    return LSTM_ERR_ALIGN;
  if (T == 0 || B == 0) return LSTM_OK;
  if ((rc = device_ok())) return rc;
  ScoreArgs a = {};
  a.x = logits; a.ld = ld; a.label = label; a.lens = seq_lens; a.stats_in = (const float2*)stats; a.entropy_in = entropy; a.dlogp = dlogp; a.dent = dent;
  a.dx = dlogits; a.ldd = ldd; a.T = T; a.B = B; a.V = V;
  a.parts = cdiv(V, 256 * kBwdPieces * (dtype == LSTM_F32 ? 4 : 8));
  if ((long)T * B * a.parts >= 1L << 24) return LSTM_ERR_DIM;       // (the threads of a launch)
  const auto kernel = dtype == LSTM_F32 ? (streams<float>(a) ? label_score_bwd_kernel<float, true> : label_score_bwd_kernel<float, false>)
                                        : (streams<bf16_t>(a) ? label_score_bwd_kernel<bf16_t, true> : label_score_bwd_kernel<bf16_t, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(T * B * a.parts)), dim3(256), 0, (hipStream_t)stream, a);
  return hipGetLastError() == hipSuccess ? LSTM_OK : LSTM_ERR_HIP;
}

}  // extern "C"
