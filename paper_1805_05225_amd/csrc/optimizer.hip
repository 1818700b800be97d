// The update of a model's weights: the global norm of the gradients, and AdamW over many tensors at once with states in 32 or 8 bits.
//
// Both are passes over memory.  The tensors' addresses travel in the launch's arguments (kItems of them, further launches take the
// rest), so nothing is copied to the device, a captured call holds its own table and two calls share nothing.
#include <math.h>
#include <algorithm>

#include "../../include/lstm_abi.h"
#include "common.h"

namespace lstm {
namespace {

constexpr int kBlock = 256;           // elements that share a scale: one wavefront's, four a lane
constexpr int kTile = 4096;           // elements of a work-group of the update: four blocks a wavefront
constexpr int kNormTile = 16384;      // elements whose squares a work-group adds
constexpr float kTop8 = 448.f;        // the largest e4m3 value

// ---- the norm ---------------------------------------------------------------------------------------------------------------
constexpr int kNormItems = 160;
struct NormArgs {
  struct Item { const void* g; long n; unsigned first; int bf16; } item[kNormItems];
  double* part;                       // one per work-group
  int count;
};
__device__ __forceinline__ double add_all(double v, double* red) {      // the sum over a work-group of four wavefronts, in thread 0
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return threadIdx.x == 0 ? (red[0] + red[1]) + (red[2] + red[3]) : 0.0;
}
__global__ __launch_bounds__(256) void grad_norm_kernel(NormArgs a) {
  __shared__ double red[4];
  int i = 0;
  for (int hi = a.count; hi - i > 1;) {
    const int mid = (i + hi) / 2;
    if (blockIdx.x >= a.item[mid].first) i = mid; else hi = mid;
  }
  const NormArgs::Item it = a.item[i];
  const long begin = (long)(blockIdx.x - it.first) * kNormTile, end = min(it.n, begin + kNormTile);
  double s = 0.0;
  for (long k = begin + threadIdx.x; k < end; k += 256) {
    const double g = it.bf16 ? Store<bf16_t>::load(it.g, k) : Store<float>::load(it.g, k);
    s += g * g;
  }
  s = add_all(s, red);
  if (threadIdx.x == 0) a.part[blockIdx.x] = s;
}
__global__ __launch_bounds__(256) void grad_norm_sum_kernel(const double* __restrict__ part, long count, float max_norm, float* __restrict__ out) {
  __shared__ double red[4];
  double s = 0.0;
  for (long k = threadIdx.x; k < count; k += 256) s += part[k];
  s = add_all(s, red);
  if (threadIdx.x == 0) {
    const double norm = sqrt(s);
    out[0] = (float)norm;
    out[1] = norm - norm != 0.0 ? __builtin_nanf("") : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
  }
}

// ---- AdamW ------------------------------------------------------------------------------------------------------------------
constexpr int kItems = 44;
struct AdamArgs {
  struct Item {
    void* p; float* w; const void* g; void* m; void* v; float* ms; float* vs;
    long n; float decay; unsigned first; int p_bf16, g_bf16;
  } item[kItems];
  int count, step;
  double lr, beta1, beta2;
  float b1, nb1, b2, nb2, eps, rate, root2;        // beta, 1 - beta; lr / (1 - beta1^t) and sqrt(1 - beta2^t) unless lr or the step is in device memory
  const float* lr_dev; const int* step_dev; const float* grad_scale;
};
static_assert(sizeof(AdamArgs) <= 4096 && sizeof(NormArgs) <= 4096, "arguments of a launch");

// beta^t in 64 bits by repeated squaring: the same on the host and on the device
__host__ __device__ inline double power(double beta, int t) {
  double r = 1.0;
  for (; t > 0; t >>= 1, beta *= beta)
    if (t & 1) r *= beta;
  return r;
}

__host__ __device__ inline void corrections(double lr, double beta1, double beta2, int t, float& rate, float& root2) {
  rate = (float)(lr / (1.0 - power(beta1, t)));
  root2 = (float)sqrt(1.0 - power(beta2, t));
}

__device__ __forceinline__ float wave_most(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}
__device__ __forceinline__ float unit8(float x, float scale) {            // x in units of the block's scale
  const float q = x / scale;
  return x == 0.f ? 0.f : q != q ? q : fminf(fmaxf(q, -kTop8), kTop8);    // (0 / 0 where a block is all zeros; a NaN stays one)
}

template <bool EIGHT>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a) {
#pragma clang fp contract(off)                                            // every product and sum rounded by itself, as the formula is written
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  if (gs - gs != 0.f) return;                                             // NaN or infinite: the step is passed over
  int i = 0;
  for (int hi = a.count; hi - i > 1;) {
    const int mid = (i + hi) / 2;
    if (blockIdx.x >= a.item[mid].first) i = mid; else hi = mid;
  }
  const AdamArgs::Item& it = a.item[i];
  const double lr = a.lr_dev ? (double)*a.lr_dev : a.lr;
  float rate = a.rate, root2 = a.root2;
  if (a.lr_dev || a.step_dev) corrections(lr, a.beta1, a.beta2, a.step_dev ? max(*a.step_dev, 1) : a.step, rate, root2);
  const float keep = (float)(1.0 - lr * it.decay);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int r = 0; r < kTile / kBlock / 4; ++r) {
    const long block = (long)(blockIdx.x - it.first) * (kTile / kBlock) + r * 4 + wave, at = block * kBlock + 4 * lane;
    if (block * kBlock >= it.n) return;
    const float ms = EIGHT ? it.ms[block] : 1.f, vs = EIGHT ? it.vs[block] : 1.f;
    float w[4], m[4], v[4], root[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      w[k] = m[k] = v[k] = root[k] = 0.f;
      if (at + k >= it.n) continue;
      w[k] = it.w ? it.w[at + k] : it.p_bf16 ? Store<bf16_t>::load(it.p, at + k) : Store<float>::load(it.p, at + k);
      const float g = (it.g_bf16 ? Store<bf16_t>::load(it.g, at + k) : Store<float>::load(it.g, at + k)) * gs;
      if (EIGHT) {
        m[k] = __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t*)it.m)[at + k], 0) * ms;
        const float old = __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t*)it.v)[at + k], 0) * vs;
        v[k] = old * old;
      } else {
        m[k] = ((const float*)it.m)[at + k];
        v[k] = ((const float*)it.v)[at + k];
      }
      m[k] = m[k] * a.b1 + g * a.nb1;
      v[k] = v[k] * a.b2 + (g * a.nb2) * g;
      root[k] = sqrtf(v[k]);
      w[k] = w[k] * keep - (m[k] / (root[k] / root2 + a.eps)) * rate;
      if (it.w) it.w[at + k] = w[k];
      if (it.p_bf16) Store<bf16_t>::store(it.p, at + k, w[k]);
      else Store<float>::store(it.p, at + k, w[k]);
      if (!EIGHT) {
        ((float*)it.m)[at + k] = m[k];
        ((float*)it.v)[at + k] = v[k];
      }
    }
    if (EIGHT) {
      float top_m = 0.f, top_r = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) { top_m = fmaxf(top_m, fabsf(m[k])); top_r = fmaxf(top_r, root[k]); }
      const float new_ms = wave_most(top_m) * (1.f / kTop8), new_vs = wave_most(top_r) * (1.f / kTop8);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (at + k >= it.n) continue;
        const int cm = __builtin_amdgcn_cvt_pk_fp8_f32(unit8(m[k], new_ms), 0.f, 0, false);
        int cv = __builtin_amdgcn_cvt_pk_fp8_f32(unit8(root[k], new_vs), 0.f, 0, false) & 255;
        if (cv == 0 && root[k] > 0.f) cv = 1;                             // the smallest code: 2^-9
        ((uint8_t*)it.m)[at + k] = (uint8_t)cm;
        ((uint8_t*)it.v)[at + k] = (uint8_t)cv;
      }
      if (lane == 0) { it.ms[block] = new_ms; it.vs[block] = new_vs; }
    }
  }
}

int items_ok(int count, const lstm_adamw_item* items) {
  if (count < 0) return LSTM_ERR_DIM;
  if (count > 0 && !items) return LSTM_ERR_NULL;
  for (int i = 0; i < count; ++i) {
    const lstm_adamw_item& it = items[i];
    if (it.count < 0 || it.count > (1L << 40)) return LSTM_ERR_DIM;
    if (it.grad_dtype != LSTM_F32 && it.grad_dtype != LSTM_BF16_F32STATE) return LSTM_ERR_UNSUPPORTED;
    if (it.count == 0) continue;
    if (!it.grad) return LSTM_ERR_NULL;
    if ((uintptr_t)it.grad & (it.grad_dtype == LSTM_F32 ? 3 : 1)) return LSTM_ERR_ALIGN;
  }
  return LSTM_OK;
}
uint64_t norm_groups(int count, const lstm_adamw_item* items) {
  uint64_t groups = 0;
  for (int i = 0; i < count; ++i) groups += (uint64_t)((items[i].count + kNormTile - 1) / kNormTile);
  return groups;
}
bool rate_ok(double x) { return x >= 0.0 && x <= 3.4028234e38; }          // (false for NaN)

}  // namespace
}  // namespace lstm

using namespace lstm;

extern "C" {

int lstm_grad_norm_query(int count, const lstm_adamw_item* items, uint64_t* workspace_bytes) {
  if (!workspace_bytes) return LSTM_ERR_NULL;
  const int rc = items_ok(count, items);
  if (rc) return rc;
  *workspace_bytes = 256 + norm_groups(count, items) * 8;
  return LSTM_OK;
}

int lstm_grad_norm(int count, const lstm_adamw_item* items, float max_norm, float* out, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!out || !workspace) return LSTM_ERR_NULL;
  int rc = items_ok(count, items);
  if (rc) return rc;
  if (!(max_norm > 0.f)) return LSTM_ERR_DIM;
  if ((uintptr_t)out & 3) return LSTM_ERR_ALIGN;
  const uint64_t groups = norm_groups(count, items);
  if (workspace_bytes < 256 + groups * 8) return LSTM_ERR_SIZE;
  if ((rc = device_ok())) return rc;
  hipStream_t s = (hipStream_t)stream;
  double* part = (double*)(((uintptr_t)workspace + 255) / 256 * 256);
  // tensors of more work-groups than a launch may have are cut into pieces of whole tiles
  constexpr long kMost = (long)kNormTile << 24;
  NormArgs a;
  a.part = part; a.count = 0;
  unsigned first = 0;
  const auto flush = [&] {
    if (a.count > 0) hipLaunchKernelGGL(grad_norm_kernel, dim3(first), dim3(256), 0, s, a);
    a.part += first;
    a.count = 0; first = 0;
  };
  for (int i = 0; i < count; ++i)
    for (long at = 0; at < items[i].count; at += kMost) {
      if (a.count == kNormItems || first >= (1u << 24)) flush();
      const bool bf16 = items[i].grad_dtype == LSTM_BF16_F32STATE;
      const long n = std::min((long)items[i].count - at, kMost);
      a.item[a.count++] = {(const char*)items[i].grad + at * (bf16 ? 2 : 4), n, first, bf16};
      first += (unsigned)((n + kNormTile - 1) / kNormTile);
    }
  flush();
  hipLaunchKernelGGL(grad_norm_sum_kernel, dim3(1), dim3(256), 0, s, part, (long)groups, max_norm, out);
  return hipGetLastError() == hipSuccess ? LSTM_OK : LSTM_ERR_HIP;
}

int lstm_adamw_step(const lstm_adamw_desc* d, int count, const lstm_adamw_item* items, void* stream) {
  if (!d) return LSTM_ERR_NULL;
  int rc = items_ok(count, items);
  if (rc) return rc;
  if (d->state_dtype != LSTM_STATE_F32 && d->state_dtype != LSTM_STATE_8BIT) return LSTM_ERR_UNSUPPORTED;
  if ((!d->lr_dev && !rate_ok(d->lr)) || !(d->beta1 >= 0.0 && d->beta1 < 1.0) || !(d->beta2 >= 0.0 && d->beta2 < 1.0) || !rate_ok(d->eps) ||
      (!d->step_dev && d->step < 1))
    return LSTM_ERR_DIM;
  if (((uintptr_t)d->lr_dev | (uintptr_t)d->step_dev | (uintptr_t)d->grad_scale) & 3) return LSTM_ERR_ALIGN;
  const bool eight = d->state_dtype == LSTM_STATE_8BIT;
  for (int i = 0; i < count; ++i) {
    const lstm_adamw_item& it = items[i];
    if (it.param_dtype != LSTM_F32 && it.param_dtype != LSTM_BF16_F32STATE) return LSTM_ERR_UNSUPPORTED;
    if (it.reserved != 0 || (it.master && it.param_dtype == LSTM_F32)) return LSTM_ERR_UNSUPPORTED;
    if (!rate_ok(it.weight_decay)) return LSTM_ERR_DIM;
    if (it.count == 0) continue;
    if (!it.param || !it.m || !it.v || (eight && (!it.m_scale || !it.v_scale))) return LSTM_ERR_NULL;
    if (((uintptr_t)it.param & (it.param_dtype == LSTM_F32 ? 3 : 1)) || ((uintptr_t)it.master & 3) ||
        (eight ? ((uintptr_t)it.m_scale | (uintptr_t)it.v_scale) & 3 : ((uintptr_t)it.m | (uintptr_t)it.v) & 3))
      return LSTM_ERR_ALIGN;
  }
  if ((rc = device_ok())) return rc;
  AdamArgs a;
  a.count = 0;
  a.step = d->step; a.lr = d->lr; a.beta1 = d->beta1; a.beta2 = d->beta2;
  a.b1 = (float)d->beta1; a.nb1 = (float)(1.0 - d->beta1); a.b2 = (float)d->beta2; a.nb2 = (float)(1.0 - d->beta2); a.eps = (float)d->eps;
  a.lr_dev = d->lr_dev; a.step_dev = d->step_dev; a.grad_scale = d->grad_scale;
  a.rate = a.root2 = 1.f;
  if (!a.lr_dev && !a.step_dev) corrections(a.lr, a.beta1, a.beta2, a.step, a.rate, a.root2);
  unsigned first = 0;
  const auto flush = [&] {
    if (a.count > 0) hipLaunchKernelGGL(eight ? adamw_kernel<true> : adamw_kernel<false>, dim3(first), dim3(256), 0, (hipStream_t)stream, a);
    a.count = 0; first = 0;
  };
  constexpr long kMost = (long)kTile << 24;
  for (int i = 0; i < count; ++i)
    for (long at = 0; at < items[i].count; at += kMost) {
      if (a.count == kItems || first >= (1u << 24)) flush();
      const lstm_adamw_item& it = items[i];
      const bool pb = it.param_dtype == LSTM_BF16_F32STATE, gb = it.grad_dtype == LSTM_BF16_F32STATE;
      const long n = std::min((long)it.count - at, kMost), ss = at * (eight ? 1 : 4);
      a.item[a.count++] = {(char*)it.param + at * (pb ? 2 : 4), it.master ? it.master + at : nullptr, (const char*)it.grad + at * (gb ? 2 : 4),
                           (char*)it.m + ss, (char*)it.v + ss, eight ? it.m_scale + at / kBlock : nullptr, eight ? it.v_scale + at / kBlock : nullptr,
                           n, it.weight_decay, first, pb, gb};
      first += (unsigned)((n + kTile - 1) / kTile);
    }
  flush();
  return hipGetLastError() == hipSuccess ? LSTM_OK : LSTM_ERR_HIP;
}

}  // extern "C"
