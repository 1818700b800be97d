// A gated linear recurrence over time, forward and backward, masked like the LSTM layers:
//
//     f, o = sigmoid(z_f, z_o)   g = tanh(z_g)   c_t = f c_{t-1} + (1 - f) g   y_t = o c_t
//     e = carry from the later frame:  dc = dy o + e,  dz_f = dc (c_{t-1} - g) f (1 - f),  dz_g = dc (1 - f)(1 - g^2),
//     dz_o = dy c o (1 - o),  e' = f dc
//
// The forward pass keeps the state in front of every 16th valid frame and nothing else: the backward pass reads z anyway, so it
// works the 15 others out again from it instead of reading them (4 bytes per frame and unit saved twice).
#include <algorithm>

#include "../../include/lstm_abi.h"
#include "common.h"

#pragma clang fp contract(off)        // products and sums are fused where it says fma, so that the forms of a kernel give the same bits

namespace lstm {
namespace {

constexpr int kSeg = 16;              // valid frames between two kept states

// A lane's access: V values of type T in one word.
template <typename T, int V> struct Word;
template <> struct Word<float, 1> {
  static __device__ unsigned load(const void* p, long i) { return ((const unsigned*)p)[i]; }
  static __device__ float get(unsigned w, int) { return __uint_as_float(w); }
  static __device__ void store(void* p, long i, const float* v) { ((float*)p)[i] = v[0]; }
};
template <> struct Word<bf16_t, 1> {
  static __device__ unsigned load(const void* p, long i) { return (unsigned)((const uint16_t*)p)[i] << 16; }
  static __device__ float get(unsigned w, int) { return __uint_as_float(w); }
  static __device__ void store(void* p, long i, const float* v) { ((uint16_t*)p)[i] = f2bf_bits(v[0]); }
};
template <> struct Word<bf16_t, 2> {
  static __device__ unsigned load(const void* p, long i) { return *(const unsigned*)((const uint16_t*)p + i); }
  static __device__ float get(unsigned w, int k) { return __uint_as_float(k == 0 ? w << 16 : w & 0xffff0000u); }
  static __device__ void store(void* p, long i, const float* v) {
    *(unsigned*)((uint16_t*)p + i) = (unsigned)f2bf_bits(v[0]) | ((unsigned)f2bf_bits(v[1]) << 16);
  }
};

// sigmoid(x) and 1 - sigmoid(x), each with the relative accuracy of a float (a forget gate near 1 leaves 1 - f its few bits otherwise)
__device__ __forceinline__ void sigmoid_pair(float x, float& s, float& not_s) {
  const float e = __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(x)), big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
  s = x < 0.f ? small : big;                                    // (NaN: both are)
  not_s = x < 0.f ? big : small;
}
__device__ __forceinline__ float sigmoid_(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x)); }
__device__ __forceinline__ float tanh_(float x) {
  const float e = __builtin_amdgcn_exp2f(-2.8853900817779268f * fabsf(x));
  return copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e), x);
}

struct ScanArgs {
  const void* z; long ldz;
  const float* c0; const int* lens;
  void* y; long ldy;
  float* cT;
  float* kept;                        // [ceil(T / kSeg)][B][n]
  const void* dy; long lddy;
  const float* dcT;
  void* dz; long lddz;
  float* dc0;
  float* dbpart;                      // [B][3n]
  int T, B, n, direction;
};
__device__ __forceinline__ int valid_frames(const int* lens, int b, int T) {
  if (!lens) return T;
  const int L = lens[b];
  return L < 0 ? 0 : (L > T ? T : L);
}

// A lane walks V units of one row of the batch through time.
template <typename T, int V>
__global__ __launch_bounds__(64) void gated_scan_fwd_kernel(ScanArgs a) {
  typedef Word<T, V> W;
  const int b = blockIdx.y, u = (blockIdx.x * 64 + threadIdx.x) * V;
  if (u >= a.n) return;
  const int L = valid_frames(a.lens, b, a.T);
  float c[V];
#pragma unroll
  for (int k = 0; k < V; ++k) c[k] = a.c0 ? a.c0[(long)b * a.n + u + k] : 0.f;
  for (int i = 0; i < L; ++i) {
    const int t = a.direction > 0 ? i : L - 1 - i;
    if (a.kept && i % kSeg == 0) {
#pragma unroll
      for (int k = 0; k < V; ++k) a.kept[((long)(i / kSeg) * a.B + b) * a.n + u + k] = c[k];
    }
    const long row = (long)t * a.B + b;
    const unsigned zf = W::load(a.z, row * a.ldz + u), zg = W::load(a.z, row * a.ldz + a.n + u), zo = W::load(a.z, row * a.ldz + 2L * a.n + u);
    float y[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      float f, nf;
      sigmoid_pair(W::get(zf, k), f, nf);
      c[k] = fmaf(f, c[k], nf * tanh_(W::get(zg, k)));
      y[k] = sigmoid_(W::get(zo, k)) * c[k];
    }
    W::store(a.y, row * a.ldy + u, y);
  }
  float zero[V] = {};
  for (int t = L; t < a.T; ++t) W::store(a.y, ((long)t * a.B + b) * a.ldy + u, zero);
  if (a.cT) {
#pragma unroll
    for (int k = 0; k < V; ++k) a.cT[(long)b * a.n + u + k] = c[k];
  }
}

template <typename T, int V>
__global__ __launch_bounds__(64) void gated_scan_bwd_kernel(ScanArgs a) {
  typedef Word<T, V> W;
  const int b = blockIdx.y, u = (blockIdx.x * 64 + threadIdx.x) * V;
  if (u >= a.n) return;
  const int L = valid_frames(a.lens, b, a.T);
  float e[V], sum[3][V] = {};
#pragma unroll
  for (int k = 0; k < V; ++k) e[k] = a.dcT ? a.dcT[(long)b * a.n + u + k] : 0.f;
  for (int q = (L + kSeg - 1) / kSeg - 1; q >= 0; --q) {
    float before[kSeg][V], c[V];
#pragma unroll
    for (int k = 0; k < V; ++k) c[k] = a.kept[((long)q * a.B + b) * a.n + u + k];
#pragma unroll
    for (int j = 0; j < kSeg; ++j) {
      const int i = min(q * kSeg + j, L - 1), t = a.direction > 0 ? i : L - 1 - i;
      const long at = ((long)t * a.B + b) * a.ldz + u;
      const unsigned zf = W::load(a.z, at), zg = W::load(a.z, at + a.n);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float f, nf;
        sigmoid_pair(W::get(zf, k), f, nf);
        before[j][k] = c[k];
        c[k] = fmaf(f, c[k], nf * tanh_(W::get(zg, k)));
      }
    }
#pragma unroll
    for (int j = kSeg - 1; j >= 0; --j) {
      const int i = q * kSeg + j, t = a.direction > 0 ? i : L - 1 - i;
      if (i < L) {
        const long row = (long)t * a.B + b, at = row * a.ldz + u, to = row * a.lddz + u;
        const unsigned zf = W::load(a.z, at), zg = W::load(a.z, at + a.n), zo = W::load(a.z, at + 2L * a.n), wy = W::load(a.dy, row * a.lddy + u);
        float df[V], dg[V], dout[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
          float f, nf, o, no;
          sigmoid_pair(W::get(zf, k), f, nf);
          sigmoid_pair(W::get(zo, k), o, no);
          const float g = tanh_(W::get(zg, k)), dy = W::get(wy, k), now = fmaf(f, before[j][k], nf * g), dc = fmaf(dy, o, e[k]);
          df[k] = dc * (before[j][k] - g) * f * nf;
          dg[k] = dc * nf * fmaf(-g, g, 1.f);
          dout[k] = dy * now * o * no;
          e[k] = f * dc;
          sum[0][k] += df[k]; sum[1][k] += dg[k]; sum[2][k] += dout[k];
        }
        W::store(a.dz, to, df);
        W::store(a.dz, to + a.n, dg);
        W::store(a.dz, to + 2L * a.n, dout);
      }
    }
  }
  float zero[V] = {};
  for (int t = L; t < a.T; ++t)
    for (int gate = 0; gate < 3; ++gate) W::store(a.dz, ((long)t * a.B + b) * a.lddz + (long)gate * a.n + u, zero);
#pragma unroll
  for (int k = 0; k < V; ++k) {
    if (a.dc0) a.dc0[(long)b * a.n + u + k] = e[k];
    if (a.dbpart)
      for (int gate = 0; gate < 3; ++gate) a.dbpart[((long)b * 3 + gate) * a.n + u + k] = sum[gate][k];
  }
}

// db = the sum of B rows of partial sums
__global__ void scan_db_kernel(const float* __restrict__ part, float* __restrict__ db, int B, int n3) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n3) return;
  float s = 0.f;
  for (int b = 0; b < B; ++b) s += part[(long)b * n3 + i];
  db[i] = s;
}

// Whole words of two values?
bool words(int n, std::initializer_list<long> ld, std::initializer_list<const void*> p) {
  uintptr_t at = 0;
  long all = n;
  for (long l : ld) all |= l;
  for (const void* q : p) at |= (uintptr_t)q;
  return (all & 1) == 0 && (at & 3) == 0;
}

int scan_dims(int T, int B, int n) {
  if (T < 0 || B < 0 || n < 1 || B > 65535 || (long)T * B > 0x7fffffffL || (long)B * n > 0x7fffffffL / 3) return LSTM_ERR_DIM;
  return LSTM_OK;
}
uint64_t reserve_need(int T, int B, int n) { return (uint64_t)((T + kSeg - 1L) / kSeg) * B * n * 4 + 256; }
uint64_t workspace_need(int B, int n) { return (uint64_t)B * n * 3 * 4 + 256; }
int scan_kind(int dtype, int direction, int T, int B, int n) {
  const int rc = scan_dims(T, B, n);
  if (rc) return rc;
  if (direction != 1 && direction != -1) return LSTM_ERR_DIRECTION;
  if (dtype != LSTM_F32 && dtype != LSTM_BF16_F32STATE) return LSTM_ERR_UNSUPPORTED;
  return LSTM_OK;
}
template <typename P> P* aligned(P* p) { return (P*)(((uintptr_t)p + 255) / 256 * 256); }

}  // namespace
}  // namespace lstm

using namespace lstm;

extern "C" {

int lstm_gated_scan_query(int T, int B, int n, uint64_t* reserve_bytes, uint64_t* workspace_bytes) {
  if (!reserve_bytes || !workspace_bytes) return LSTM_ERR_NULL;
  const int rc = scan_dims(T, B, n);
  if (rc) return rc;
  *reserve_bytes = reserve_need(T, B, n);
  *workspace_bytes = workspace_need(B, n);
  return LSTM_OK;
}

int lstm_gated_scan_fwd(int dtype, int direction, int T, int B, int n, const void* z, int64_t ldz, const float* c0, const int32_t* seq_lens,
                        void* y, int64_t ldy, float* cT, void* reserve, uint64_t reserve_bytes, void* workspace, uint64_t workspace_bytes,
                        void* stream) {
  if (((!z || !y) && T > 0 && B > 0) || !workspace) return LSTM_ERR_NULL;      // (arrays without elements may have no address)
  int rc = scan_kind(dtype, direction, T, B, n);
  if (rc) return rc;
  if (ldz < 3L * n || ldy < n) return LSTM_ERR_DIM;
  if ((((uintptr_t)z | (uintptr_t)y) & (dtype == LSTM_F32 ? 3 : 1)) || (((uintptr_t)c0 | (uintptr_t)seq_lens | (uintptr_t)cT | (uintptr_t)reserve) & 3))
    return LSTM_ERR_ALIGN;
  if ((reserve && reserve_bytes < reserve_need(T, B, n)) || workspace_bytes < workspace_need(B, n)) return LSTM_ERR_SIZE;
  if (B == 0) return LSTM_OK;
  if ((rc = device_ok())) return rc;
  ScanArgs a = {};
  a.z = z; a.ldz = ldz; a.c0 = c0; a.lens = seq_lens; a.y = y; a.ldy = ldy; a.cT = cT; a.kept = reserve ? aligned((float*)reserve) : nullptr;
  a.T = T; a.B = B; a.n = n; a.direction = direction;
  const int V = dtype == LSTM_BF16_F32STATE && words(n, {ldz, ldy}, {z, y}) ? 2 : 1;
  const auto kernel = dtype == LSTM_F32 ? gated_scan_fwd_kernel<float, 1> : V == 2 ? gated_scan_fwd_kernel<bf16_t, 2> : gated_scan_fwd_kernel<bf16_t, 1>;
  hipLaunchKernelGGL(kernel,
                     dim3(cdiv(n, 64 * V), B), dim3(64), 0, (hipStream_t)stream, a);
  return hipGetLastError() == hipSuccess ? LSTM_OK : LSTM_ERR_HIP;
}

int lstm_gated_scan_bwd(int dtype, int direction, int T, int B, int n, const void* z, int64_t ldz, const int32_t* seq_lens, const void* reserve,
                        uint64_t reserve_bytes, const void* dy, int64_t lddy, const float* dcT, void* dz, int64_t lddz, float* dc0, float* db,
                        void* workspace, uint64_t workspace_bytes, void* stream) {
  if (((!z || !dy || !dz) && T > 0 && B > 0) || !reserve || !workspace) return LSTM_ERR_NULL;
  int rc = scan_kind(dtype, direction, T, B, n);
  if (rc) return rc;
  if (ldz < 3L * n || lddy < n || lddz < 3L * n) return LSTM_ERR_DIM;
  if ((((uintptr_t)z | (uintptr_t)dy | (uintptr_t)dz) & (dtype == LSTM_F32 ? 3 : 1)) ||
      (((uintptr_t)seq_lens | (uintptr_t)reserve | (uintptr_t)dcT | (uintptr_t)dc0 | (uintptr_t)db) & 3))
    return LSTM_ERR_ALIGN;
  if (reserve_bytes < reserve_need(T, B, n) || workspace_bytes < workspace_need(B, n)) return LSTM_ERR_SIZE;
  if (B == 0 && !db) return LSTM_OK;
  if ((rc = device_ok())) return rc;
  hipStream_t s = (hipStream_t)stream;
  ScanArgs a = {};
  a.z = z; a.ldz = ldz; a.lens = seq_lens; a.kept = (float*)aligned((const float*)reserve); a.dy = dy; a.lddy = lddy; a.dcT = dcT; a.dz = dz; a.lddz = lddz;
  a.dc0 = dc0; a.dbpart = db ? aligned((float*)workspace) : nullptr;
  a.T = T; a.B = B; a.n = n; a.direction = direction;
  const int V = dtype == LSTM_BF16_F32STATE && words(n, {ldz, lddy, lddz}, {z, dy, dz}) ? 2 : 1;
  const auto kernel = dtype == LSTM_F32 ? gated_scan_bwd_kernel<float, 1> : V == 2 ? gated_scan_bwd_kernel<bf16_t, 2> : gated_scan_bwd_kernel<bf16_t, 1>;
  if (B > 0)
    hipLaunchKernelGGL(kernel,
                       dim3(cdiv(n, 64 * V), B), dim3(64), 0, s, a);
  if (db) hipLaunchKernelGGL(scan_db_kernel, dim3(cdiv(3L * n, 256)), dim3(256), 0, s, a.dbpart, db, B, 3 * n);
  return hipGetLastError() == hipSuccess ? LSTM_OK : LSTM_ERR_HIP;
}

}  // extern "C"
