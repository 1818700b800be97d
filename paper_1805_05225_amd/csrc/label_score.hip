// Log probabilities of given labels under the softmax of an output layer's logits, with entropy, best alternatives and gradient:
//
//     m = max x,  z = sum e^(x - m)      logp = (x[label] - m) - log z      entropy = log z - (sum e^(x - m) (x - m)) / z
//     dlogits[v] = dlogp ([v = label] - p[v]) - dent p[v] (log p[v] + entropy),  log p = (x - m) - log z
//
// m, z and u = sum e^(x - m) (x - m) are kept running: where m grows by d, z' = z e^-d and u' = (u - d z) e^-d.
#include <algorithm>

#include "../../include/lstm_abi.h"
#include "common.h"

#pragma clang fp contract(off)        // products and sums are fused where it says fma, so that the forms of a kernel give the same bits

namespace lstm {
namespace {

constexpr int kTopMax = 16;
constexpr int kVocabMost = 1 << 26;

struct ScoreArgs {
  const void* x; long ld;
  const int* label; const int* lens;
  float* logp; float* entropy; float2* stats;
  float* top_logp; int* top_label;
  const float2* stats_in; const float* entropy_in; const float* dlogp; const float* dent;
  void* dx; long ldd;
  int T, B, V, top;
};
__device__ __forceinline__ bool padded(const ScoreArgs& a, int r) { return a.lens && r / a.B >= a.lens[r % a.B]; }

// What a row's exponentials add up to relative to m; -inf, 0, 0 is the empty sum.
struct Sums { float m, z, u; };
__device__ __forceinline__ float base_of(float m) { return fmaxf(m, -__FLT_MAX__); }    // (no -inf - -inf)
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b) {
  Sums c;
  c.m = fmaxf(a.m, b.m);
  const float base = base_of(c.m), da = fmaxf(base_of(a.m) - base, -1.0e4f), db = fmaxf(base_of(b.m) - base, -1.0e4f), ea = __expf(da), eb = __expf(db);
  c.z = a.z * ea + b.z * eb;
  c.u = (a.u + da * a.z) * ea + (b.u + db * b.z) * eb;
  return c;
}
__device__ __forceinline__ void add(Sums& s, float x) {
  if (x == -__builtin_inff()) return;
  const Sums one = {x, x - x == 0.f ? 1.f : __builtin_nanf(""), 0.f};                   // NaN and +inf: no sum
  s = join(s, one);
}

// A work-group per row.
template <typename T>
__global__ __launch_bounds__(256) void label_score_kernel(ScoreArgs a) {
  __shared__ Sums part[4];
  __shared__ float win_v[4];
  __shared__ int win_i[4];
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float kNegInf = -__builtin_inff();
  const bool pad = padded(a, r);
  const T* row = (const T*)a.x + (long)r * a.ld;
  Sums s = {kNegInf, 0.f, 0.f};
  if (!pad)
    for (int v = tid; v < a.V; v += 256) add(s, Store<T>::load(row, v));
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const Sums other = {__shfl_xor(s.m, o), __shfl_xor(s.z, o), __shfl_xor(s.u, o)};
    s = join(s, other);
  }
  if (lane == 0) part[wave] = s;
  __syncthreads();
  s = join(join(part[0], part[1]), join(part[2], part[3]));
  const float logz = logf(s.z);
  if (tid == 0) {
    if (a.stats) a.stats[r] = pad ? make_float2(0.f, 0.f) : s.z == 0.f ? make_float2(kNegInf, 0.f) : make_float2(s.m, logz);
    if (a.entropy) a.entropy[r] = pad || s.z == 0.f ? 0.f : logz - s.u / s.z;
    if (a.logp) {
      const int l = a.label[r];
      float p = 0.f;
      if (!pad && l >= 0 && l < a.V) {
        const float x = Store<T>::load(row, l);
        p = s.z == 0.f ? kNegInf : (x - s.m) - logz;
      }
      a.logp[r] = p;
    }
  }
  float last_v = __builtin_inff();
  int last_i = -1;
  for (int k = 0; k < a.top; ++k) {                                      // every thread offers its best behind the last winner
    float bv = kNegInf;
    int bi = 0x7fffffff;
    if (!pad && logz - logz == 0.f)
      for (int v = tid; v < a.V; v += 256) {
        const float x = Store<T>::load(row, v);
        if ((x < last_v || (x == last_v && v > last_i)) && (x > bv)) { bv = x; bi = v; }
      }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const float ov = __shfl_xor(bv, o);
      const int oi = __shfl_xor(bi, o);
      if (ov > bv || (ov == bv && oi < bi)) { bv = ov; bi = oi; }
    }
    if (lane == 0) { win_v[wave] = bv; win_i[wave] = bi; }
    __syncthreads();
    for (int w = 0; w < 4; ++w)
      if (win_v[w] > bv || (win_v[w] == bv && win_i[w] < bi)) { bv = win_v[w]; bi = win_i[w]; }
    __syncthreads();
    if (tid == 0) {
      a.top_logp[(long)r * a.top + k] = bi == 0x7fffffff ? kNegInf : (bv - s.m) - logz;
      a.top_label[(long)r * a.top + k] = bi == 0x7fffffff ? 0 : bi;
    }
    last_v = bv;
    last_i = bi;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void label_score_bwd_kernel(ScoreArgs a) {
  const int r = blockIdx.x;
  const bool pad = padded(a, r);
  const T* row = (const T*)a.x + (long)r * a.ld;
  T* out = (T*)a.dx + (long)r * a.ldd;
  const int l = a.dlogp && !pad ? a.label[r] : -1;
  const float dl = l >= 0 && l < a.V ? a.dlogp[r] : 0.f, de = a.dent && !pad ? a.dent[r] : 0.f, h = a.dent && !pad ? a.entropy_in[r] : 0.f;
  const float2 st = pad ? make_float2(0.f, 0.f) : a.stats_in[r];
  const bool none = pad || (dl == 0.f && de == 0.f) || st.x == -__builtin_inff();
  for (int v = threadIdx.x; v < a.V; v += 256) {
    float d = 0.f;
    if (!none) {
      const float x = Store<T>::load(row, v), q = (x - st.x) - st.y, p = __expf(q);
      d = fmaf(-p, fmaf(de, fmaxf(q, -1.0e4f) + h, dl), v == l ? dl : 0.f);
    }
    Store<T>::store(out, v, d);
  }
}

int score_dims(int T, int B, int V, int top) {
  if (T < 0 || B < 0 || V < 1 || top < 0 || (long)T * B > 0x7fffffffL / 16) return LSTM_ERR_DIM;
  if (V > kVocabMost || top > kTopMax) return LSTM_ERR_UNSUPPORTED;
  return LSTM_OK;
}

}  // namespace
}  // namespace lstm

using namespace lstm;

extern "C" {

int lstm_label_score_query(int T, int B, int V, int top, uint64_t* workspace_bytes) {
  if (!workspace_bytes) return LSTM_ERR_NULL;
  const int rc = score_dims(T, B, V, top);
  if (rc) return rc;
  *workspace_bytes = 256;
  return LSTM_OK;
}

int lstm_label_score_fwd(int dtype, int T, int B, int V, const void* logits, int64_t ld, const int32_t* label, const int32_t* seq_lens,
                         float* logp, float* entropy, float* stats, int top, float* top_logp, int32_t* top_label, void* workspace,
                         uint64_t workspace_bytes, void* stream) {
  const bool any = T > 0 && B > 0;                             // (arrays without elements may have no address)
  if (!workspace || (any && (!logits || (logp && !label) || (top > 0 && (!top_logp || !top_label))))) return LSTM_ERR_NULL;
  int rc = score_dims(T, B, V, top);
  if (rc) return rc;
  if (ld < V) return LSTM_ERR_DIM;
  if (dtype != LSTM_F32 && dtype != LSTM_BF16_F32STATE) return LSTM_ERR_UNSUPPORTED;
  if (((uintptr_t)logits & (dtype == LSTM_F32 ? 3 : 1)) || (((uintptr_t)label | (uintptr_t)seq_lens | (uintptr_t)logp | (uintptr_t)entropy |
      (uintptr_t)top_logp | (uintptr_t)top_label) & 3) || ((uintptr_t)stats & 7))
    return LSTM_ERR_ALIGN;
  uint64_t need = 0;
  lstm_label_score_query(T, B, V, top, &need);
  if (workspace_bytes < need) return LSTM_ERR_SIZE;
  if (T == 0 || B == 0) return LSTM_OK;
  if ((rc = device_ok())) return rc;
  ScoreArgs a = {};
  a.x = logits; a.ld = ld; a.label = label; a.lens = seq_lens; a.logp = logp; a.entropy = entropy; a.stats = (float2*)stats; a.top = top; a.top_logp = top_logp;
  a.top_label = top_label; a.T = T; a.B = B; a.V = V;
  hipLaunchKernelGGL(dtype == LSTM_F32 ? label_score_kernel<float> : label_score_kernel<bf16_t>, dim3((unsigned)(T * B)), dim3(256), 0, (hipStream_t)stream, a);
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
  hipLaunchKernelGGL(dtype == LSTM_F32 ? label_score_bwd_kernel<float> : label_score_bwd_kernel<bf16_t>, dim3((unsigned)(T * B)), dim3(256), 0, (hipStream_t)stream, a);
  return hipGetLastError() == hipSuccess ? LSTM_OK : LSTM_ERR_HIP;
}

}  // extern "C"
