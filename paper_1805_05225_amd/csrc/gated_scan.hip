// A gated linear recurrence over time, forward and backward, masked like the LSTM layers:
//
//     f, o = sigmoid(z_f, z_o)   g = tanh(z_g)   c_t = f c_{t-1} + (1 - f) g   y_t = o c_t
//     e = carry from the later frame:  dc = dy o + e,  dz_f = dc (c_{t-1} - g) f (1 - f),  dz_g = dc (1 - f)(1 - g^2),
//     dz_o = dy c o (1 - o),  e' = f dc
//
// The forward pass keeps the state in front of every 16th (few frames: 8th) valid frame and nothing else: the backward pass reads z anyway, so it
// works the others out again from it instead of reading them (4 bytes per frame and unit saved twice).
#include <algorithm>

#include "../../include/lstm_abi.h"
#include "common.h"
#include "exchange_dev.h"

#pragma clang fp contract(off)        // products and sums are fused where it says fma, so that the forms of a kernel give the same bits (where time is cut at the same frames)

namespace lstm {
namespace {

constexpr int kWaves = 8;             // wavefronts of a work-group at most
// Valid frames of a wavefront in a round, and between two kept states.  16 fill a lane's registers; short batches take 8, so that more wavefronts share
// them and more of these fit a compute unit (80 frames of 64 rows of 1000 bfloat16 values, backward: 26 us with 16, 20 with 8; 512 of 64 rows of 2048 213 and 219).
constexpr int kSeg = 16, kSegShort = 8, kShort = 128;
inline int seg_of(int T) { return T <= kShort ? kSegShort : kSeg; }

// A lane's access: V values of type T in one word, `at` bytes into a row.  A row is a buffer of its own: its address stays in scalar registers, and
// what lies outside (a lane behind the last unit, a frame that is not there) is read as 0 and not written, without a branch.
typedef __amdgpu_buffer_rsrc_t Row;
constexpr unsigned kOutside = 0x80000000u;
constexpr int kLine = 128;              // bytes of a line of the L2 cache
constexpr int kNonTemporal = 2;         // cache policy of a load: past the caches
template <typename T, int V> struct Word;
template <> struct Word<float, 1> {
  template <int POLICY> static __device__ unsigned load(Row r, unsigned at) { return __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, POLICY); }
  static __device__ float get(unsigned w, int) { return __uint_as_float(w); }
  static __device__ void store(Row r, unsigned at, const float* v) { __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[0]), r, at, 0, 0); }
  static constexpr unsigned kInf = 0x7f800000u;
};
template <> struct Word<bf16_t, 1> {
  template <int POLICY> static __device__ unsigned load(Row r, unsigned at) { return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, at, 0, POLICY); }
  static __device__ float get(unsigned w, int) { return __uint_as_float(w << 16); }      // (not in load, which would wait there)
  static __device__ void store(Row r, unsigned at, const float* v) { __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, (bf16_t)v[0]), r, at, 0, 0); }
  static constexpr unsigned kInf = 0x7f80u;
};
template <> struct Word<bf16_t, 2> {
  typedef __attribute__((ext_vector_type(2))) float f2;
  typedef __attribute__((ext_vector_type(2))) bf16_t b2;
  template <int POLICY> static __device__ unsigned load(Row r, unsigned at) { return __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, POLICY); }
  static __device__ float get(unsigned w, int k) { return __uint_as_float(k == 0 ? w << 16 : w & 0xffff0000u); }
  static __device__ void store(Row r, unsigned at, const float* v) {        // rounded to nearest, ties to even
    const f2 x = {v[0], v[1]};
    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, __builtin_convertvector(x, b2)), r, at, 0, 0);
  }
  static constexpr unsigned kInf = 0x7f807f80u;
};

// The same behind an address of the lane's own.
template <typename T, int V> __device__ __forceinline__ unsigned word_at(const void* p, long i) {
  if constexpr (sizeof(T) * V == 4) return *(const unsigned*)((const T*)p + i);
  else return *((const uint16_t*)p + i);
}

// sigmoid(x) and 1 - sigmoid(x) with e = exp(-x): 1 / (1 + e) and e / (1 + e), each with a float's relative accuracy (1 - f has few bits left
// where a forget gate is near 1) down to 2^-126, below which the hardware's reciprocal and exponential give 0.  The reciprocal does so where e, still finite or not, is above
// 2^126 (x < -87.33), and e / (1 + e) is 1 there.  A NaN stays in both.
__device__ __forceinline__ void sigmoid_pair(float x, float& s, float& not_s) {
  const float e = __builtin_amdgcn_exp2f(-1.4426950408889634f * x);
  s = __builtin_amdgcn_rcpf(1.f + e);
  not_s = e >= 0x1p126f ? 1.f : e * s;
}
__device__ __forceinline__ float sigmoid_(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x)); }
// tanh(x) = 1 - 2 / (1 + exp(2 x)) is off by up to 2^-23 of 1, so it keeps few digits of a small value.  In float storage the Taylor series takes its place near 0 (the
// first term left out is 9e-9 of it at 1/4; 32768 x 1 x 1024 154 -> 158 us forward, 263 -> 265 backward).  With bfloat16 values of z, 2^-9 of themselves apart, that
// is a relative error of the same size only below 2^-14, and the series would cost 8 % of a call of 1500 x 32 x 1024.
template <typename T> __device__ __forceinline__ float tanh_(float x) {
  const float far = fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(2.8853900817779268f * x)), 1.f);
  if constexpr (sizeof(T) == 2) return far;
  const float q = x * x, near = fmaf(x * q, fmaf(q, fmaf(q, fmaf(q, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), x);
  return fabsf(x) < 0.25f ? near : far;
}

struct ScanArgs {
  const void* z; long ldz;
  const float* c0; const int* lens;
  void* y; long ldy;
  float* cT;
  float* kept;                        // [ceil(T / seg_of(T))][B][n]
  const void* dy; long lddy;
  const float* dcT;
  void* dz; long lddz;
  float* dc0;
  float* dbpart;                      // [parts * B][3n]
  float2* join;                       // [parts][B][n]: what a part's frames do to a state, (factor, addend)
  float* first;                       // [B][n]: copy of c0 or dcT
  int T, B, n, direction;
  bool shared;                        // columns of a row share lines of 128 bytes
  int parts, per;                     // time is cut into parts of `per` valid frames (a multiple of a work-group's round)
};
__device__ __forceinline__ int valid_frames(const int* lens, int b, int T) {
  if (!lens) return T;
  const int L = __builtin_amdgcn_readfirstlane(lens[b]);
  return L < 0 ? 0 : (L > T ? T : L);
}
// The valid frames of a part, as numbers in the order of the walk, and where their rows lie.
struct Span {
  int L, begin, end;
  long row0; int step;                // row of walk number i: row0 + i * step
  __device__ __forceinline__ Span(const ScanArgs& a, int b, int part) {
    L = valid_frames(a.lens, b, a.T);
    begin = part * a.per;
    end = min(L, begin + a.per);
    row0 = a.direction > 0 ? b : (long)(L - 1) * a.B + b;
    step = a.direction > 0 ? a.B : -a.B;
  }
};
// Consecutive rows of the walk from number `first` on; `bytes`: what of a row is there.
template <typename T> struct Rows {
  const char* p; long stride; int bytes;
  __device__ __forceinline__ Rows(const void* base, long ld, const Span& sp, int first, int columns)
      : p((const char*)base + (sp.row0 + (long)first * sp.step) * ld * (long)sizeof(T)), stride(sp.step * ld * (long)sizeof(T)), bytes(columns * (int)sizeof(T)) {}
  __device__ __forceinline__ Row row(bool there = true) const { return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, there ? bytes : 0, kBufFlags); }
  __device__ __forceinline__ void next() { p += stride; }
  __device__ __forceinline__ void back() { p -= stride; }
};
template <typename T> __device__ __forceinline__ Row row_at(const void* base, long row, long ld, int columns) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)base + row * ld * (long)sizeof(T)), 0, columns * (int)sizeof(T), kBufFlags);
}

// Which columns (in work-groups), row of the batch and part a work-group takes.  Work-groups go to the eight XCDs in turn; all columns of a row go to one of them, so that
// the lines where one work-group's units end and the next one's begin meet in its L2 instead of being read, and written in pieces, by two (with the note on non-temporal loads below:
// 2000 frames of 32 rows of 1000 bfloat16 values 130 -> 118 us forward, 311 -> 226 backward; 1024, whose lines are nobody else's, 112 and 202 without it, 113 and 209 with it).
struct Place {
  int x, b, part;
  __device__ __forceinline__ explicit Place(bool shared) {
    unsigned row = blockIdx.y + gridDim.y * blockIdx.z, column = blockIdx.x;
    if (shared && row < ((gridDim.y * gridDim.z) & ~7u)) {
      const unsigned id = column + gridDim.x * row, turn = id >> 3;
      row = turn / gridDim.x;
      column = turn - row * gridDim.x;
      row = row * 8 + (id & 7);
    }
    row = __builtin_amdgcn_readfirstlane(row);
    x = __builtin_amdgcn_readfirstlane(column);
    part = __builtin_amdgcn_readfirstlane(row / gridDim.y);
    b = (int)row - part * (int)gridDim.y;
  }
};

// What a work-group's wavefronts tell each other: the composition of their frames, c -> A c + C, for every unit; two sets, so that one
// barrier a round is enough.
template <int V, int NW> struct Chain { float a[2][NW][V][64], c[2][NW][V][64]; };

// The state that enters wavefront `wave`'s frames and the one that leaves all of them, from `state` and the compositions of the nw <= NW wavefronts.  order: 1 if
// wavefront 0 comes first, -1 if it comes last.
template <int V, int NW>
__device__ __forceinline__ void link(Chain<V, NW>& s, int set, int lane, int wave, int nw, int order, const float (&A)[V], const float (&C)[V],
                                     float (&state)[V], float (&mine)[V]) {
#pragma unroll
  for (int k = 0; k < V; ++k) { s.a[set][wave][k][lane] = A[k]; s.c[set][wave][k][lane] = C[k]; }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    const int w = order > 0 ? i : NW - 1 - i;
    if (w >= nw) continue;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (w == wave) mine[k] = state[k];
      state[k] = fmaf(s.a[set][w][k][lane], state[k], s.c[set][w][k][lane]);
    }
  }
}

// A work-group takes 64 V units of one row of the batch through a part of time, NW * SEG frames a round: every wavefront has SEG of them in
// registers, composes them into one step c -> A c + C, gets the state that enters them from the others' compositions and walks them
// with it.  So all loads of a round are in flight together, z is read once and only the compositions cross wavefronts.  80 frames of 64 rows of 1000 bfloat16 values, lengths
// 20 to 80: 12 us, a round or two, latency; 1500 of 32 rows of 1024, lengths 200 to 1500: 83 (264 MB), the longest rows' work-groups; 32768 of one row of 1024 float, with the
// compositions of its parts: 147 (797 MB, 5.4 TB/s), memory and, before the first round, the parts in front folded one behind the other.  (In replayed graphs, without a profiler.)
template <typename T, int V, int NW, int SEG, bool STREAM>
__global__ __launch_bounds__(64 * NW, 4) void gated_scan_fwd_kernel(ScanArgs a) {
  typedef Word<T, V> W;
  __shared__ Chain<V, NW> chain;
  const Place place(a.shared);
  const int b = place.b, part = a.parts - 1 - place.part, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nw = (int)blockDim.x >> 6;
  const int u = (place.x * 64 + lane) * V;
  const bool live = u < a.n;
  const int at = live ? u : 0;
  const unsigned o0 = live ? at * (unsigned)sizeof(T) : kOutside, o1 = o0 + a.n * (unsigned)sizeof(T), o2 = o1 + a.n * (unsigned)sizeof(T);
  const Span sp(a, b, part);
  const float* c0 = a.parts > 1 ? a.first : a.c0;
  float c[V];
#pragma unroll
  for (int k = 0; k < V; ++k) c[k] = c0 ? c0[(long)b * a.n + at + k] : 0.f;
  if (sp.begin < sp.L)
    for (int p = 0; p < part; ++p)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float2 j = a.join[((long)p * a.B + b) * a.n + at + k];
        c[k] = fmaf(j.x, c[k], j.y);
      }
  int set = 0;
  for (int base = sp.begin; base < sp.end; base += nw * SEG, set ^= 1) {
    const int s0 = base + wave * SEG, count = min(SEG, sp.end - s0);
    float f[SEG][V], add[SEG][V], A[V], C[V], mine[V];
    unsigned zo[SEG];
#pragma unroll
    for (int k = 0; k < V; ++k) { A[k] = 1.f; C[k] = 0.f; }
    if (count > 0) {
      unsigned zf[SEG], zg[SEG];
      Rows<T> z(a.z, a.ldz, sp, s0, 3 * a.n);
#pragma unroll
      for (int j = 0; j < SEG; ++j, z.next()) {
        const Row r = z.row(j < count);
        zf[j] = W::template load<STREAM ? kNonTemporal : 0>(r, o0);
        zg[j] = W::template load<STREAM ? kNonTemporal : 0>(r, o1);
        zo[j] = W::template load<STREAM ? kNonTemporal : 0>(r, o2);
      }
#pragma unroll
      for (int j = 0; j < SEG; ++j) {
        if (j >= count) zf[j] = W::kInf;                         // f = 1 and 1 - f = 0: the state stays
#pragma unroll
        for (int k = 0; k < V; ++k) {
          float nf;
          sigmoid_pair(W::get(zf[j], k), f[j][k], nf);
          add[j][k] = nf * tanh_<T>(W::get(zg[j], k));
          A[k] *= f[j][k];
          C[k] = fmaf(f[j][k], C[k], add[j][k]);
        }
      }
    }
    link<V, NW>(chain, set, lane, wave, nw, 1, A, C, c, mine);
    if (count > 0) {
      if (a.kept && live) {
#pragma unroll
        for (int k = 0; k < V; ++k) a.kept[((long)(s0 / SEG) * a.B + b) * a.n + u + k] = mine[k];
      }
      Rows<T> to(a.y, a.ldy, sp, s0, a.n);
#pragma unroll
      for (int j = 0; j < SEG; ++j, to.next()) {
        float y[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
          mine[k] = fmaf(f[j][k], mine[k], add[j][k]);
          y[k] = sigmoid_(W::get(zo[j], k)) * mine[k];
        }
        W::store(to.row(j < count), o0, y);
      }
    }
  }
  if (!live) return;
  const float zero[V] = {};
  for (int t = sp.L + part * nw + wave; t < a.T; t += a.parts * nw) W::store(row_at<T>(a.y, (long)t * a.B + b, a.ldy, a.n), o0, zero);
  if (a.cT && wave == 0 && (sp.L == 0 ? part == 0 : (sp.L - 1) / a.per == part)) {
#pragma unroll
    for (int k = 0; k < V; ++k) a.cT[(long)b * a.n + u + k] = c[k];
  }
}

// One frame (or none), the step of a search or of generation: nothing to compose, a lane per word of any row.  (As a stretch of one frame of the kernel above,
// a wavefront per row and 64 words: 768 rows of 1000 bfloat16 values 6.2 us, 4.4 so.)
template <typename T, int V>
__global__ __launch_bounds__(256) void gated_scan_step_kernel(ScanArgs a) {
  typedef Word<T, V> W;
  const unsigned i = blockIdx.x * 256 + threadIdx.x, per_row = (unsigned)(a.n / V);
  if (i >= per_row * (unsigned)a.B) return;
  const int b = (int)(i / per_row), u = (int)(i - (unsigned)b * per_row) * V;
  const long state = (long)b * a.n + u, row = (long)b * a.ldz + u;
  float c[V], y[V];
#pragma unroll
  for (int k = 0; k < V; ++k) c[k] = a.c0 ? a.c0[state + k] : 0.f;
  const bool valid = a.T > 0 && (!a.lens || a.lens[b] > 0);
  if (valid) {
    const unsigned zf = word_at<T, V>(a.z, row), zg = word_at<T, V>(a.z, row + a.n), zo = word_at<T, V>(a.z, row + 2L * a.n);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (a.kept) a.kept[state + k] = c[k];
      float f, nf;
      sigmoid_pair(W::get(zf, k), f, nf);
      c[k] = fmaf(f, c[k], nf * tanh_<T>(W::get(zg, k)));
      y[k] = sigmoid_(W::get(zo, k)) * c[k];
    }
  }
  if (a.T > 0) {
#pragma unroll
    for (int k = 0; k < V; ++k) ((T*)a.y)[(long)b * a.ldy + u + k] = (T)(valid ? y[k] : 0.f);
  }
  if (a.cT) {
#pragma unroll
    for (int k = 0; k < V; ++k) a.cT[state + k] = c[k];
  }
}

// The compositions of all parts but the last, for the kernel above, and a copy of c0 (which cT may overwrite while other parts read it).
template <typename T, int V, int NW, int SEG, bool STREAM>
__global__ __launch_bounds__(64 * NW, 4) void gated_scan_join_kernel(ScanArgs a) {
  typedef Word<T, V> W;
  __shared__ Chain<V, NW> chain;
  const Place place(a.shared);
  const int b = place.b, part = place.part, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int u = (place.x * 64 + lane) * V;
  const bool live = u < a.n;
  const int at = live ? u : 0;
  const unsigned o0 = live ? at * (unsigned)sizeof(T) : kOutside, o1 = o0 + a.n * (unsigned)sizeof(T), o2 = o1 + a.n * (unsigned)sizeof(T);
  const Span sp(a, b, part);
  if (part == 0 && live && wave == 0) {
#pragma unroll
    for (int k = 0; k < V; ++k) a.first[(long)b * a.n + u + k] = a.c0 ? a.c0[(long)b * a.n + u + k] : 0.f;
  }
  float A[V], C[V];
#pragma unroll
  for (int k = 0; k < V; ++k) { A[k] = 1.f; C[k] = 0.f; }
  for (int base = sp.begin; base < sp.end; base += NW * SEG) {
    // each wavefront composes consecutive frames of its own eighth of the part
    const int eighth = a.per / NW, from = sp.begin + wave * eighth, s0 = from + (base - sp.begin) / NW, count = min(SEG, min(sp.end, from + eighth) - s0);
    if (count <= 0) break;
    unsigned zf[SEG], zg[SEG];
    Rows<T> z(a.z, a.ldz, sp, s0, 3 * a.n);
#pragma unroll
    for (int j = 0; j < SEG; ++j, z.next()) {
      const Row r = z.row(j < count);
      zf[j] = W::template load<STREAM ? kNonTemporal : 0>(r, o0);
      zg[j] = W::template load<STREAM ? kNonTemporal : 0>(r, o1);
    }
#pragma unroll
    for (int j = 0; j < SEG; ++j) {
      if (j >= count) zf[j] = W::kInf;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float f, nf;
        sigmoid_pair(W::get(zf[j], k), f, nf);
        A[k] *= f;
        C[k] = fmaf(f, C[k], nf * tanh_<T>(W::get(zg[j], k)));
      }
    }
  }
#pragma unroll
  for (int k = 0; k < V; ++k) { chain.a[0][wave][k][lane] = A[k]; chain.c[0][wave][k][lane] = C[k]; }
  __syncthreads();
  if (wave != 0 || !live) return;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float2 j = make_float2(1.f, 0.f);
    for (int w = 0; w < NW; ++w) {
      j.x *= chain.a[0][w][k][lane];
      j.y = fmaf(chain.a[0][w][k][lane], j.y, chain.c[0][w][k][lane]);
    }
    a.join[((long)part * a.B + b) * a.n + u + k] = j;
  }
}

// The same from the other end.  A wavefront works its SEG states out again from the one that the forward pass kept in front of them; what
// passes on is e = f dc, whose frames compose like the forward ones: e -> A e + C with A = the product of f.  The calls above, with the sum of db: 19, 128 (519 MB) and
// 256 us (1330 MB with the compositions, 5.2 TB/s).
template <typename T, int V, int NW, int SEG, bool STREAM>
__global__ __launch_bounds__(64 * NW, SEG == kSeg && sizeof(T) == 2 ? 2 : 4) void gated_scan_bwd_kernel(ScanArgs a) {
  typedef Word<T, V> W;
  __shared__ union { Chain<V, NW> chain; double sum[NW][3][V][64]; } sh;
  const Place place(a.shared);
  const int b = place.b, part = a.parts - 1 - place.part, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nw = (int)blockDim.x >> 6;
  const int u = (place.x * 64 + lane) * V;
  const bool live = u < a.n;
  const int at = live ? u : 0;
  const unsigned o0 = live ? at * (unsigned)sizeof(T) : kOutside, o1 = o0 + a.n * (unsigned)sizeof(T), o2 = o1 + a.n * (unsigned)sizeof(T);
  const Span sp(a, b, part);
  float e[V];
  double total[3][V] = {};
#pragma unroll
  for (int k = 0; k < V; ++k) e[k] = a.dcT ? a.dcT[(long)b * a.n + at + k] : 0.f;
  if (sp.begin < sp.L)
    for (int p = (sp.L - 1) / a.per; p > part; --p)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float2 j = a.join[((long)p * a.B + b) * a.n + at + k];
        e[k] = fmaf(j.x, e[k], j.y);
      }
  int set = 0;
  for (int base = sp.begin + (sp.end - 1 - sp.begin) / (nw * SEG) * (nw * SEG); sp.begin < sp.end && base >= sp.begin; base -= nw * SEG, set ^= 1) {
    const int s0 = base + wave * SEG, count = min(SEG, sp.end - s0);
    float f[SEG][V], nf[SEG][V], g[SEG][V], o[SEG][V], c[SEG + 1][V], A[V], C[V], mine[V];      // c[j], c[j + 1]: the state before and behind frame j
    unsigned wy[SEG];
#pragma unroll
    for (int k = 0; k < V; ++k) { A[k] = 1.f; C[k] = 0.f; }
    if (count > 0) {
      unsigned zf[SEG], zg[SEG], zo[SEG];
#pragma unroll
      for (int k = 0; k < V; ++k) c[0][k] = a.kept[((long)(s0 / SEG) * a.B + b) * a.n + at + k];
      Rows<T> z(a.z, a.ldz, sp, s0, 3 * a.n), dy(a.dy, a.lddy, sp, s0, a.n);
#pragma unroll
      for (int j = 0; j < SEG; ++j, z.next(), dy.next()) {
        const Row r = z.row(j < count);
        zf[j] = W::template load<STREAM ? kNonTemporal : 0>(r, o0);
        zg[j] = W::template load<STREAM ? kNonTemporal : 0>(r, o1);
        zo[j] = W::template load<STREAM ? kNonTemporal : 0>(r, o2);
        wy[j] = W::template load<STREAM ? kNonTemporal : 0>(dy.row(j < count), o0);
      }
#pragma unroll
      for (int j = 0; j < SEG; ++j) {
        if (j >= count) zf[j] = W::kInf;                         // f = 1, 1 - f = 0 (and dy = 0): e stays
#pragma unroll
        for (int k = 0; k < V; ++k) {
          sigmoid_pair(W::get(zf[j], k), f[j][k], nf[j][k]);
          g[j][k] = tanh_<T>(W::get(zg[j], k));
          o[j][k] = sigmoid_(W::get(zo[j], k));
          c[j + 1][k] = fmaf(f[j][k], c[j][k], nf[j][k] * g[j][k]);
        }
      }
#pragma unroll
      for (int j = SEG - 1; j >= 0; --j)
#pragma unroll
        for (int k = 0; k < V; ++k) {
          A[k] *= f[j][k];
          C[k] = f[j][k] * fmaf(W::get(wy[j], k), o[j][k], C[k]);
        }
    }
    link<V, NW>(sh.chain, set, lane, wave, nw, -1, A, C, e, mine);
    if (count > 0) {
      float sum[3][V] = {};
      Rows<T> to(a.dz, a.lddz, sp, s0 + SEG - 1, 3 * a.n);
#pragma unroll
      for (int j = SEG - 1; j >= 0; --j, to.back()) {
        float df[V], dg[V], dout[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float dy = W::get(wy[j], k), dc = fmaf(dy, o[j][k], mine[k]);
          mine[k] = f[j][k] * dc;
          df[k] = (c[j][k] - g[j][k]) * nf[j][k] * mine[k];
          dg[k] = dc * nf[j][k] * fmaf(-g[j][k], g[j][k], 1.f);
          dout[k] = dy * c[j + 1][k] * fmaf(-o[j][k], o[j][k], o[j][k]);
          sum[0][k] += df[k]; sum[1][k] += dg[k]; sum[2][k] += dout[k];
        }
        const Row r = to.row(j < count);
        W::store(r, o0, df);
        W::store(r, o1, dg);
        W::store(r, o2, dout);
      }
#pragma unroll
      for (int gate = 0; gate < 3; ++gate)
#pragma unroll
        for (int k = 0; k < V; ++k) total[gate][k] += (double)sum[gate][k];
    }
  }
  if (live) {
    const float zero[V] = {};
    for (int t = sp.L + part * nw + wave; t < a.T; t += a.parts * nw) {
      const Row r = row_at<T>(a.dz, (long)t * a.B + b, a.lddz, 3 * a.n);
      W::store(r, o0, zero);
      W::store(r, o1, zero);
      W::store(r, o2, zero);
    }
    if (a.dc0 && part == 0 && wave == 0) {
#pragma unroll
      for (int k = 0; k < V; ++k) a.dc0[(long)b * a.n + u + k] = e[k];
    }
  }
  if (!a.dbpart) return;
  __syncthreads();                                              // (the chain's memory is used again)
#pragma unroll
  for (int gate = 0; gate < 3; ++gate)
#pragma unroll
    for (int k = 0; k < V; ++k) sh.sum[wave][gate][k][lane] = total[gate][k];
  __syncthreads();
  if (!live || wave != 0) return;
  for (int gate = 0; gate < 3; ++gate)
#pragma unroll
    for (int k = 0; k < V; ++k) {
      double d = 0.0;
      for (int w = 0; w < nw; ++w) d += sh.sum[w][gate][k][lane];
      a.dbpart[(((long)part * a.B + b) * 3 + gate) * a.n + u + k] = (float)d;
    }
}

// The backward compositions of all parts but the first.
template <typename T, int V, int NW, int SEG, bool STREAM>
__global__ __launch_bounds__(64 * NW, 4) void gated_scan_bwd_join_kernel(ScanArgs a) {
  typedef Word<T, V> W;
  __shared__ Chain<V, NW> chain;
  const Place place(a.shared);
  const int b = place.b, part = place.part + 1, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int u = (place.x * 64 + lane) * V;
  const bool live = u < a.n;
  const int at = live ? u : 0;
  const unsigned o0 = live ? at * (unsigned)sizeof(T) : kOutside, o1 = o0 + a.n * (unsigned)sizeof(T), o2 = o1 + a.n * (unsigned)sizeof(T);
  const Span sp(a, b, part);
  float A[V], C[V];
#pragma unroll
  for (int k = 0; k < V; ++k) { A[k] = 1.f; C[k] = 0.f; }
  const int eighth = a.per / NW, from = sp.begin + wave * eighth, to = min(sp.end, from + eighth);
  for (int s0 = from + (eighth / SEG - 1) * SEG; s0 >= from; s0 -= SEG) {
    const int count = min(SEG, to - s0);
    if (count <= 0) continue;
    unsigned zf[SEG], zo[SEG], wy[SEG];
    Rows<T> z(a.z, a.ldz, sp, s0, 3 * a.n), dy(a.dy, a.lddy, sp, s0, a.n);
#pragma unroll
    for (int j = 0; j < SEG; ++j, z.next(), dy.next()) {
      const Row r = z.row(j < count);
      zf[j] = W::template load<STREAM ? kNonTemporal : 0>(r, o0);
      zo[j] = W::template load<STREAM ? kNonTemporal : 0>(r, o2);
      wy[j] = W::template load<STREAM ? kNonTemporal : 0>(dy.row(j < count), o0);
    }
#pragma unroll
    for (int j = SEG - 1; j >= 0; --j) {
      if (j >= count) zf[j] = W::kInf;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float f = sigmoid_(W::get(zf[j], k));
        A[k] *= f;
        C[k] = f * fmaf(W::get(wy[j], k), sigmoid_(W::get(zo[j], k)), C[k]);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < V; ++k) { chain.a[0][wave][k][lane] = A[k]; chain.c[0][wave][k][lane] = C[k]; }
  __syncthreads();
  if (wave != 0 || !live) return;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float2 j = make_float2(1.f, 0.f);
    for (int w = NW - 1; w >= 0; --w) {
      j.x *= chain.a[0][w][k][lane];
      j.y = fmaf(chain.a[0][w][k][lane], j.y, chain.c[0][w][k][lane]);
    }
    a.join[((long)part * a.B + b) * a.n + u + k] = j;
  }
}

// db = the sum of `rows` rows of partial sums (each added in 64 bits and rounded once): 64 columns a work-group, whose wavefronts share the rows
constexpr int kDbWaves = 16;
__global__ __launch_bounds__(64 * kDbWaves) void scan_db_kernel(const float* __restrict__ part, float* __restrict__ db, int rows, int n3) {
  __shared__ double sum[kDbWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x * 64 + lane;
  double s = 0.0;
  if (i < n3)
    for (int r = wave; r < rows; r += 8 * kDbWaves) {             // eight loads in flight
      float x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = part[(long)min(r + k * kDbWaves, rows - 1) * n3 + i];
#pragma unroll
      for (int k = 0; k < 8; ++k) s += r + k * kDbWaves < rows ? (double)x[k] : 0.0;
    }
  sum[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || i >= n3) return;
  for (int w = 1; w < kDbWaves; ++w) s += sum[w][lane];
  db[i] = (float)s;
}

// Does every gate of every row start at a multiple of `bytes`?
bool starts_at(uintptr_t bytes, int size, int n, std::initializer_list<long> ld, std::initializer_list<const void*> p) {
  uintptr_t all = (uintptr_t)n * size;
  for (long l : ld) all |= (uintptr_t)l * size;
  for (const void* q : p) all |= (uintptr_t)q;
  return all % bytes == 0;
}

int scan_dims(int T, int B, int n) {
  if (T < 0 || T > (1 << 30) || B < 0 || n < 1 || n > (1 << 27) || B > 65535 || (long)T * B > 0x7fffffffL || (long)B * n > 0x7fffffffL / 3) return LSTM_ERR_DIM;
  return LSTM_OK;
}
uint64_t reserve_need(int T, int B, int n) { return (uint64_t)cdiv(T, seg_of(T)) * B * n * 4 + 256; }

// How the work is cut.  (Where time is cut decides how compositions are grouped, and so the last bits of results.  Only for long texts of few rows, below, does that depend on V, and with it on the
// addresses of rows: 32768 bfloat16 frames of 2 rows of 512 at odd elements, cut as often as those at whole words, take 112 us forward instead of 95 and 163 backward instead of 153.)
// Short batches have work-groups of fewer wavefronts; where rows and units give too few work-groups for the device, time is cut
// into parts, whose compositions a launch before works out (a second reading of two thirds of what the forward pass reads, three quarters of the
// backward pass).
struct Cut { int V, waves, parts, per; };
Cut cut_of(int T, int B, int n, int V) {
  // Single values instead of words where these give few work-groups: 2048 frames of 16 rows of 1024 87 -> 69 us forward, 147 -> 109 backward; 2048 of 2 rows of 512
  // 22 -> 16 and 29 -> 21.  Not where time is cut either way and long enough to be cut as often as one likes (words against single values, forward and backward: 16384 of 1, 4 and 8 rows
  // of 1024 53, 89 and 51, 87; 156, 269 and 172, 296; 311, 520 and 332, 565; 65536 of 1 row 163, 278 and 175, 302, but of 256 units, where the fold of 128 parts counts, 95, 132 and 68, 97;
  // beside the rule 8192 of 2 rows 47, 88 and 48, 85, of 8 rows 155, 265 and 165, 287, 16384 of 16 rows 666, 1060 and 487, 865).
  const long wide_groups = (long)cdiv(n, 128) * B;
  if (T > 1 && wide_groups < 256 && !(T >= 16384 && wide_groups <= 64)) V = 1;
  Cut c = {V, std::max(1, std::min(kWaves, cdiv(T, seg_of(T)))), 1, std::max(T, 1)};
  const long groups = (long)cdiv(n, 64 * V) * B;
  // Time is cut up to 128 work-groups, half the compute units: with more the second reading costs more than the idle units (uncut and cut, forward and backward, float rows of 1024:
  // 4096 of 10 rows 158, 267 and 184, 319; of 16 219, 404 and 265, 482; 8192 of 10 322, 532 and 393, 629; 1024 of 10 44, 69 and 51, 80).
  constexpr long kGroups = 512;
  const int round = kWaves * kSeg;
  if (groups > 0 && groups <= 128 && T >= 4 * round) {
    c.per = cdiv(cdiv(T, (int)std::min(kGroups / groups, (long)T / (2 * round))), round) * round;
    c.parts = cdiv(T, c.per);
  }
  return c;
}
// What the parts of a call leave each other in the workspace.
struct Places { uint64_t join, first, dbpart, total; };
Places places_of(int T, int B, int n, bool backward) {           // (for either width of a word: the rows' addresses decide which is used)
  const auto up = [](uint64_t x) { return (x + 255) / 256 * 256; };
  const uint64_t parts = std::max(cut_of(T, B, n, 1).parts, cut_of(T, B, n, 2).parts), state = (uint64_t)B * n * 4;
  Places p;
  p.join = 0;
  p.first = parts > 1 ? up(parts * state * 2) : 0;
  p.dbpart = p.first + (parts > 1 ? up(state) : 0);
  p.total = p.dbpart + (backward ? up(parts * state * 3) : 0);
  if (p.total > 0) p.total += 256;
  return p;
}
uint64_t workspace_need(int T, int B, int n, bool backward) { return places_of(T, B, n, backward).total; }
int scan_kind(int dtype, int direction, int T, int B, int n) {
  const int rc = scan_dims(T, B, n);
  if (rc) return rc;
  if (direction != 1 && direction != -1) return LSTM_ERR_DIRECTION;
  if (dtype != LSTM_F32 && dtype != LSTM_BF16_F32STATE) return LSTM_ERR_UNSUPPORTED;
  return LSTM_OK;
}
template <typename P> P* aligned(P* p) { return (P*)(((uintptr_t)p + 255) / 256 * 256); }
void place(ScanArgs& a, const Cut& c, void* workspace, bool backward) {
  const Places p = places_of(a.T, a.B, a.n, backward);
  char* ws = aligned((char*)workspace);
  a.join = (float2*)(ws + p.join); a.first = (float*)(ws + p.first); a.dbpart = (float*)(ws + p.dbpart);
  a.parts = c.parts; a.per = c.per;
}
int status() { return hipGetLastError() == hipSuccess ? LSTM_OK : LSTM_ERR_HIP; }

// STREAM: a call that moves more than the last-level cache holds (us, 32768 x 1 x 1024 float 167 -> 153 forward and 275 -> 261 backward, 512 x 64 x 2048 bfloat16 121 -> 110
// forward, 1500 x 32 x 1024 141 -> 125 backward; 80 x 64 x 1000, which fits, 19 -> 23 backward), of rows whose work-groups share no lines: those are to stay in L2 for the
// neighbour (2000 x 32 x 1000 bfloat16 120 -> 118 forward, 276 -> 226 backward without it).
template <typename T, int V, bool STREAM>
int run_fwd(const ScanArgs& a, const Cut& c, hipStream_t s) {
  const dim3 grid(cdiv(a.n, 64 * V), a.B, c.parts), most(grid.x, grid.y, c.parts - 1);
  if (c.parts > 1) {
    const auto join = gated_scan_join_kernel<T, V, kWaves, kSeg, STREAM>;
    hipLaunchKernelGGL(join, most, dim3(64 * kWaves), 0, s, a);
  }
  // A single work-group a compute unit is twice as wide: 1500 frames of 32 rows of 1024 bfloat16 values 92 us with eight wavefronts, 84 with sixteen.
  const bool wide = c.waves == kWaves && c.parts == 1 && a.T >= 2 * kWaves * kSeg && (long)grid.x * a.B < 512;
  const auto kernel = a.T <= kShort ? gated_scan_fwd_kernel<T, V, kWaves, kSegShort, STREAM>
                      : wide ? gated_scan_fwd_kernel<T, V, 2 * kWaves, kSeg, STREAM> : gated_scan_fwd_kernel<T, V, kWaves, kSeg, STREAM>;
  hipLaunchKernelGGL(kernel, grid, dim3(64 * (wide ? 2 * kWaves : c.waves)), 0, s, a);
  return status();
}
template <typename T, int V, bool STREAM>
int run_bwd(const ScanArgs& a, const Cut& c, float* db, hipStream_t s) {
  const dim3 grid(cdiv(a.n, 64 * V), a.B, c.parts), most(grid.x, grid.y, c.parts - 1);
  if (c.parts > 1) {
    const auto join = gated_scan_bwd_join_kernel<T, V, kWaves, kSeg, STREAM>;
    hipLaunchKernelGGL(join, most, dim3(64 * kWaves), 0, s, a);
  }
  const auto kernel = a.T <= kShort ? gated_scan_bwd_kernel<T, V, kWaves, kSegShort, STREAM> : gated_scan_bwd_kernel<T, V, kWaves, kSeg, STREAM>;
  if (a.B > 0) hipLaunchKernelGGL(kernel, grid, dim3(64 * c.waves), 0, s, a);
  if (db) hipLaunchKernelGGL(scan_db_kernel, dim3(cdiv(3L * a.n, 64)), dim3(64 * kDbWaves), 0, s, a.dbpart, db, c.parts * a.B, 3 * a.n);
  return status();
}
bool streams(const ScanArgs& a, int size, int values) { return !a.shared && (uint64_t)a.T * a.B * a.n * size * values > kLastLevelBytes; }      // values: a unit's, of a frame
template <typename T, int V>
int run_fwd(const ScanArgs& a, const Cut& c, hipStream_t s) {
  if (a.T <= 1) {
    hipLaunchKernelGGL((gated_scan_step_kernel<T, V>), dim3(cdiv((long)(a.n / V) * a.B, 256)), dim3(256), 0, s, a);
    return status();
  }
  return streams(a, sizeof(T), 4) ? run_fwd<T, V, true>(a, c, s) : run_fwd<T, V, false>(a, c, s);
}
template <typename T, int V>
int run_bwd(const ScanArgs& a, const Cut& c, float* db, hipStream_t s) {
  return streams(a, sizeof(T), 7) ? run_bwd<T, V, true>(a, c, db, s) : run_bwd<T, V, false>(a, c, db, s);
}

}  // namespace
}  // namespace lstm

using namespace lstm;

extern "C" {

int lstm_gated_scan_query(int T, int B, int n, uint64_t* reserve_bytes, uint64_t* fwd_workspace_bytes, uint64_t* bwd_workspace_bytes) {
  if (!reserve_bytes || !fwd_workspace_bytes || !bwd_workspace_bytes) return LSTM_ERR_NULL;
  const int rc = scan_dims(T, B, n);
  if (rc) return rc;
  *reserve_bytes = reserve_need(T, B, n);
  *fwd_workspace_bytes = workspace_need(T, B, n, false);
  *bwd_workspace_bytes = workspace_need(T, B, n, true);
  return LSTM_OK;
}

int lstm_gated_scan_fwd(int dtype, int direction, int T, int B, int n, const void* z, int64_t ldz, const float* c0, const int32_t* seq_lens,
                        void* y, int64_t ldy, float* cT, void* reserve, uint64_t reserve_bytes, void* workspace, uint64_t workspace_bytes,
                        void* stream) {
  if ((!z || !y) && T > 0 && B > 0) return LSTM_ERR_NULL;        // (arrays without elements may have no address)
  int rc = scan_kind(dtype, direction, T, B, n);
  if (rc) return rc;
  if (ldz < 3L * n || ldy < n) return LSTM_ERR_DIM;
  if ((((uintptr_t)z | (uintptr_t)y) & (dtype == LSTM_F32 ? 3 : 1)) || (((uintptr_t)c0 | (uintptr_t)seq_lens | (uintptr_t)cT | (uintptr_t)reserve) & 3))
    return LSTM_ERR_ALIGN;
  const uint64_t need = workspace_need(T, B, n, false);
  if (need > 0 && !workspace) return LSTM_ERR_NULL;
  if ((reserve && reserve_bytes < reserve_need(T, B, n)) || workspace_bytes < need) return LSTM_ERR_SIZE;
  if (B == 0) return LSTM_OK;
  if ((rc = device_ok())) return rc;
  ScanArgs a = {};
  a.z = z; a.ldz = ldz; a.c0 = c0; a.lens = seq_lens; a.y = y; a.ldy = ldy; a.cT = cT; a.kept = reserve ? aligned((float*)reserve) : nullptr;
  a.T = T; a.B = B; a.n = n; a.direction = direction;
  const int size = dtype == LSTM_F32 ? 4 : 2;
  a.shared = !starts_at(kLine, size, n, {ldz, ldy}, {z, y});
  const Cut c = cut_of(T, B, n, size == 2 && starts_at(4, size, n, {ldz, ldy}, {z, y}) ? 2 : 1);
  place(a, c, workspace, false);
  return dtype == LSTM_F32 ? run_fwd<float, 1>(a, c, (hipStream_t)stream) : c.V == 2 ? run_fwd<bf16_t, 2>(a, c, (hipStream_t)stream) : run_fwd<bf16_t, 1>(a, c, (hipStream_t)stream);
}

int lstm_gated_scan_bwd(int dtype, int direction, int T, int B, int n, const void* z, int64_t ldz, const int32_t* seq_lens, const void* reserve,
                        uint64_t reserve_bytes, const void* dy, int64_t lddy, const float* dcT, void* dz, int64_t lddz, float* dc0, float* db,
                        void* workspace, uint64_t workspace_bytes, void* stream) {
  if (((!z || !dy || !dz) && T > 0 && B > 0) || !reserve) return LSTM_ERR_NULL;
  int rc = scan_kind(dtype, direction, T, B, n);
  if (rc) return rc;
  if (ldz < 3L * n || lddy < n || lddz < 3L * n) return LSTM_ERR_DIM;
  if ((((uintptr_t)z | (uintptr_t)dy | (uintptr_t)dz) & (dtype == LSTM_F32 ? 3 : 1)) ||
      (((uintptr_t)seq_lens | (uintptr_t)reserve | (uintptr_t)dcT | (uintptr_t)dc0 | (uintptr_t)db) & 3))
    return LSTM_ERR_ALIGN;
  const uint64_t need = workspace_need(T, B, n, true);
  if (need > 0 && !workspace) return LSTM_ERR_NULL;
  if (reserve_bytes < reserve_need(T, B, n) || workspace_bytes < need) return LSTM_ERR_SIZE;
  if (B == 0 && !db) return LSTM_OK;
  if ((rc = device_ok())) return rc;
  hipStream_t s = (hipStream_t)stream;
  ScanArgs a = {};
  a.z = z; a.ldz = ldz; a.lens = seq_lens; a.kept = (float*)aligned((const float*)reserve); a.dy = dy; a.lddy = lddy; a.dcT = dcT; a.dz = dz; a.lddz = lddz;
  a.dc0 = dc0; a.T = T; a.B = B; a.n = n; a.direction = direction;
  const int size = dtype == LSTM_F32 ? 4 : 2;
  a.shared = !starts_at(kLine, size, n, {ldz, lddy, lddz}, {z, dy, dz});
  const Cut c = cut_of(T, B, n, size == 2 && starts_at(4, size, n, {ldz, lddy, lddz}, {z, dy, dz}) ? 2 : 1);
  place(a, c, workspace, true);
  if (!db) a.dbpart = nullptr;
  return dtype == LSTM_F32 ? run_bwd<float, 1>(a, c, db, s) : c.V == 2 ? run_bwd<bf16_t, 2>(a, c, db, s) : run_bwd<bf16_t, 1>(a, c, db, s);
}

}  // extern "C"
