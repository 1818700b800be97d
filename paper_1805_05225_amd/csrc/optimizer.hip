// The update of a model's weights: the global norm of the gradients, and AdamW over many tensors at once with states in 32 or 8 bits.
//
// Both are passes over memory.  The tensors' addresses travel in the launch's arguments (as many as these hold, further launches take the
// rest), so nothing is copied to the device, the update needs no workspace, a captured call holds its own table and two calls share nothing.
#include <math.h>
#include <algorithm>

#include "../../include/lstm_abi.h"
#include "common.h"

namespace lstm {
namespace {

constexpr int kBlock = 256;           // elements that share a scale: one wavefront's, four a lane
constexpr int kTile = 1024;           // elements of a work-group of the update: a block a wavefront
constexpr int kNormTile = 16384;      // elements whose squares a work-group adds
constexpr float kTop8 = 448.f;        // the largest e4m3 value

// ---- the norm ---------------------------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
constexpr int kNormItems = 254;       // (16 bytes each: what 4096 bytes of a launch's arguments hold)
constexpr long kNormMost = 1L << 31;  // elements of an item
struct NormArgs {
  uint64_t g[kNormItems];             // address, and 1 if the elements are bfloat16
  unsigned n[kNormItems], first[kNormItems];
  double* part;                       // one per work-group
  int count;
};
// the item that tile t belongs to, from the items' first tiles
__device__ __forceinline__ int find(const unsigned* first, int count, unsigned t) {
  int i = 0;
  for (int hi = count; hi - i > 1;) {
    const int mid = (i + hi) / 2;
    if (t >= first[mid]) i = mid; else hi = mid;
  }
  return i;
}
template <int NW = 4>
__device__ __forceinline__ double add_all(double v, double* red) {      // the sum over a work-group of NW wavefronts, in thread 0
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
  if (threadIdx.x == 0)
    for (int w = 0; w < NW; ++w) s += red[w];
  return s;
}
__device__ __forceinline__ void write_norm(double sum, float max_norm, float* out) {
  const double norm = sqrt(sum);
  out[0] = (float)norm;
  out[1] = norm - norm != 0.0 ? __builtin_nanf("") : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
}
// A thread's share of the sum of squares of elements [begin, end): whole pieces of 16 bytes between the first and the last such boundary, what lies
// on either side one by one.  Eight loads of a thread are in flight together.
// STREAM: past the caches, for more gradients than the last-level cache would keep for the update that follows (133 M float ones: 82 us, 6.5 TB/s).
template <int NT, bool STREAM>
__device__ __forceinline__ double squares(const void* g, long begin, long end, bool bf16, int tid) {
  double s = 0.0;
  const auto square = [&](float x) { const double d = x; s = __builtin_fma(d, d, s); };
  const int size = bf16 ? 2 : 4;
  const char* p = (const char*)g + begin * size;
  const int n = (int)(end - begin), head = min(n, (int)(-(uintptr_t)p & 15) / size), per = 16 / size, pieces = (n - head) / per, tail = n - head - pieces * per;
  if (tid < head + tail) {
    const int at = tid < head ? tid : head + pieces * per + tid - head;
    square(bf16 ? Store<bf16_t>::load(p, at) : Store<float>::load(p, at));
  }
  const u32x4* q = (const u32x4*)(p + head * size);
  constexpr int U = 8;
  for (int at = tid; at < pieces; at += U * NT) {
    u32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = at + u * NT >= pieces ? u32x4{0u, 0u, 0u, 0u} : STREAM ? __builtin_nontemporal_load(q + at + u * NT) : q[at + u * NT];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        square(__uint_as_float(bf16 ? x[u][e] << 16 : x[u][e]));
        if (bf16) square(__uint_as_float(x[u][e] & 0xffff0000u));
      }
  }
  return s;
}
template <bool STREAM>
__global__ __launch_bounds__(256) void grad_norm_kernel(NormArgs a) {
  __shared__ double red[4];
  const int i = find(a.first, a.count, blockIdx.x);
  const long begin = (long)(blockIdx.x - a.first[i]) * kNormTile, end = min((long)a.n[i], begin + kNormTile);
  const double s = add_all(squares<256, STREAM>((const void*)(a.g[i] & ~1ull), begin, end, a.g[i] & 1, threadIdx.x), red);
  if (threadIdx.x == 0) a.part[blockIdx.x] = s;
}
__global__ __launch_bounds__(1024) void grad_norm_sum_kernel(const double* __restrict__ part, long count, float max_norm, float* __restrict__ out) {
  __shared__ double red[16];
  double s = 0.0;
  for (long k = threadIdx.x; k < count; k += 1024) s += part[k];
  s = add_all<16>(s, red);
  if (threadIdx.x == 0) write_norm(s, max_norm, out);
}
// Few elements: one work-group, one launch, its wavefronts taking kNormFewTile elements each.
constexpr long kNormFew = 65536;
constexpr int kNormFewTile = 2048;
__global__ __launch_bounds__(1024) void grad_norm_few_kernel(NormArgs a, unsigned tiles, float max_norm, float* __restrict__ out) {
  __shared__ double red[16];
  double s = 0.0;
  for (unsigned t = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); t < tiles; t += 16) {
    const int i = find(a.first, a.count, t);
    const long begin = (long)(t - a.first[i]) * kNormFewTile;
    s += squares<64, false>((const void*)(a.g[i] & ~1ull), begin, min((long)a.n[i], begin + kNormFewTile), a.g[i] & 1, threadIdx.x & 63);
  }
  s = add_all<16>(s, red);
  if (threadIdx.x == 0) write_norm(s, max_norm, out);
}

// ---- AdamW ------------------------------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(4))) bf16_t bf16x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
constexpr int kItems = 58;            // (68 bytes each: likewise)
constexpr long kMost = 1L << 28;      // elements of an item
static_assert(kTile == 4 * kBlock, "a work-group has four wavefronts");
struct Item {
  void* p; float* w; const void* g; void* m; void* v; float* ms; float* vs;
  unsigned n; bool p_bf16, g_bf16, wide; float decay;
};
struct AdamArgs {
  void* p[kItems]; float* w[kItems]; const void* g[kItems]; void* m[kItems]; void* v[kItems]; float* ms[kItems]; float* vs[kItems];
  float decay[kItems];
  unsigned kind[kItems], first[kItems];            // elements * 8 + p_bf16 + 2 g_bf16 + 4 wide
  __host__ __device__ __forceinline__ void put(int i, const Item& x, unsigned at) {
    p[i] = x.p; w[i] = x.w; g[i] = x.g; m[i] = x.m; v[i] = x.v; ms[i] = x.ms; vs[i] = x.vs; decay[i] = x.decay; first[i] = at;
    kind[i] = x.n << 3 | (unsigned)x.p_bf16 | (unsigned)x.g_bf16 << 1 | (unsigned)x.wide << 2;
  }
  __device__ __forceinline__ Item get(int i) const {
    return {p[i], w[i], g[i], m[i], v[i], ms[i], vs[i], kind[i] >> 3, (kind[i] & 1) != 0, (kind[i] & 2) != 0, (kind[i] & 4) != 0, decay[i]};
  }
  int count, step;
  double lr, beta1, beta2;
  float b1, nb1, b2, nb2, eps, rate, inv_root2;    // beta, 1 - beta; lr / (1 - beta1^t) and 1 / sqrt(1 - beta2^t) unless lr or the step is in device memory
  const float* lr_dev; const int* step_dev; const float* grad_scale;
};
static_assert(sizeof(AdamArgs) <= 4096 && sizeof(NormArgs) + 16 <= 4096, "arguments of a launch");

// beta^t in 64 bits by repeated squaring: the same on the host and on the device
__host__ __device__ inline double power(double beta, int t) {
  double r = 1.0;
  for (; t > 0; t >>= 1, beta *= beta)
    if (t & 1) r *= beta;
  return r;
}

__host__ __device__ inline void corrections(double lr, double beta1, double beta2, int t, float& rate, float& inv_root2) {
  rate = (float)(lr / (1.0 - power(beta1, t)));
  inv_root2 = (float)(1.0 / sqrt(1.0 - power(beta2, t)));
}

__device__ __forceinline__ float wave_most(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}
// Four values in units of a block's scale as e4m3 codes.  The quotient is the correctly rounded one (a code that depends on the last bit of an
// approximation is another code than the formula's, and the next step sees it): from the scale's reciprocal, worked out once for the block, and
// one correction by the remainder; by a division where the reciprocal of a tiny scale is infinite, or the scale is 0.
struct Unit { float scale, inv; };
__device__ __forceinline__ Unit unit_of(float scale) {
  Unit u = {scale, __builtin_amdgcn_rcpf(scale)};
  u.inv = fmaf(fmaf(-scale, u.inv, 1.f), u.inv, u.inv);
  return u;
}
__device__ __forceinline__ unsigned pack8(const float (&x)[4], const Unit& u) {
  float q[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    q[k] = x[k] * u.inv;
    q[k] = fmaf(fmaf(-q[k], u.scale, x[k]), u.inv, q[k]);
  }
  if (!(u.scale > 1e-36f && u.scale < 1e36f)) {                            // (the same for the whole wavefront)
#pragma unroll
    for (int k = 0; k < 4; ++k) q[k] = x[k] == 0.f ? 0.f : x[k] / u.scale;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) q[k] = q[k] != q[k] ? q[k] : __builtin_amdgcn_fmed3f(q[k], -kTop8, kTop8);          // (a NaN stays one)
  return __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false), true);
}

// Four consecutive elements of an array of float or bfloat16, past the caches: each is read and written once (133 M bfloat16 weights with masters, norm included, 847 -> 759 us,
// in 8 bits 554 -> 484; nothing lost where all of it would fit the last-level cache).
__device__ __forceinline__ void load4(const void* p, bool bf16, long at, float (&x)[4]) {
  if (bf16) {
    const u32x2 w = __builtin_nontemporal_load((const u32x2*)((const uint16_t*)p + at));
    x[0] = __uint_as_float(w[0] << 16); x[1] = __uint_as_float(w[0] & 0xffff0000u);
    x[2] = __uint_as_float(w[1] << 16); x[3] = __uint_as_float(w[1] & 0xffff0000u);
  } else {
    const f32x4 w = __builtin_nontemporal_load((const f32x4*)((const float*)p + at));
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = w[k];
  }
}
__device__ __forceinline__ void store4(void* p, bool bf16, long at, const float (&x)[4]) {
  const f32x4 w = {x[0], x[1], x[2], x[3]};
  if (bf16) __builtin_nontemporal_store(__builtin_convertvector(w, bf16x4), (bf16x4*)((bf16_t*)p + at));
  else __builtin_nontemporal_store(w, (f32x4*)((float*)p + at));
}

// What a lane holds of a block of 256 elements: four consecutive ones.
template <bool EIGHT> struct Block {
  float w[4], g[4];
  float m[4], v[4];                   // (unused in 8 bits until they are worked out)
  unsigned cm, cv;
  float ms, vs;
};
// WIDE: every array of the tensor starts at a multiple of four elements' bytes, and the 256 elements are all there; otherwise element by element.
template <bool EIGHT, bool WIDE>
__device__ __forceinline__ void fetch(Block<EIGHT>& x, const Item& it, long block, int lane) {
  const long at = block * kBlock + 4 * lane;
  if (WIDE) {
    load4(it.g, it.g_bf16, at, x.g);
    if (it.w) load4(it.w, false, at, x.w); else load4(it.p, it.p_bf16, at, x.w);
    if (EIGHT) {
      x.cm = __builtin_nontemporal_load((const unsigned*)((const uint8_t*)it.m + at));
      x.cv = __builtin_nontemporal_load((const unsigned*)((const uint8_t*)it.v + at));
    } else {
      load4(it.m, false, at, x.m);
      load4(it.v, false, at, x.v);
    }
  } else {
    const int left = (int)min(4L, max(0L, (long)it.n - at));
    x.cm = x.cv = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool there = k < left;
      x.g[k] = !there ? 0.f : it.g_bf16 ? Store<bf16_t>::load(it.g, at + k) : Store<float>::load(it.g, at + k);
      x.w[k] = !there ? 0.f : it.w ? it.w[at + k] : it.p_bf16 ? Store<bf16_t>::load(it.p, at + k) : Store<float>::load(it.p, at + k);
      if (EIGHT) {
        if (there) {
          x.cm |= (unsigned)((const uint8_t*)it.m)[at + k] << (8 * k);
          x.cv |= (unsigned)((const uint8_t*)it.v)[at + k] << (8 * k);
        }
      } else {
        x.m[k] = there ? ((const float*)it.m)[at + k] : 0.f;
        x.v[k] = there ? ((const float*)it.v)[at + k] : 0.f;
      }
    }
  }
  if (EIGHT) { x.ms = it.ms[block]; x.vs = it.vs[block]; }
}
template <bool EIGHT, bool WIDE>
__device__ __forceinline__ void update(Block<EIGHT>& x, const Item& it, const AdamArgs& a, long block, int lane, float gs, float keep, float rate,
                                       float inv_root2) {
#pragma clang fp contract(off)                                            // every product and sum rounded by itself, as the formula is written
  const long at = block * kBlock + 4 * lane;
  const int left = WIDE ? 4 : (int)min(4L, max(0L, (long)it.n - at));
  float root[4];
  if (EIGHT) {
    x.m[0] = __builtin_amdgcn_cvt_f32_fp8(x.cm, 0); x.m[1] = __builtin_amdgcn_cvt_f32_fp8(x.cm, 1); x.m[2] = __builtin_amdgcn_cvt_f32_fp8(x.cm, 2); x.m[3] = __builtin_amdgcn_cvt_f32_fp8(x.cm, 3);
    x.v[0] = __builtin_amdgcn_cvt_f32_fp8(x.cv, 0); x.v[1] = __builtin_amdgcn_cvt_f32_fp8(x.cv, 1); x.v[2] = __builtin_amdgcn_cvt_f32_fp8(x.cv, 2); x.v[3] = __builtin_amdgcn_cvt_f32_fp8(x.cv, 3);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x.m[k] *= x.ms;
      x.v[k] *= x.vs;
      x.v[k] *= x.v[k];
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float g = x.g[k] * gs;
    x.m[k] = x.m[k] * a.b1 + g * a.nb1;
    x.v[k] = x.v[k] * a.b2 + (g * a.nb2) * g;
    // the quotient by the hardware's reciprocal (1 unit in the last place), the root in full (the hardware's takes a v below 2^-126 for 0).  A denominator below 2^-126, that of
    // an element without gradients where eps is that small, is moved into the range that the reciprocal has, or 0 / eps were 0 * inf
    root[k] = sqrtf(x.v[k]);
    const float den = root[k] * inv_root2 + a.eps, up = den < 0x1p-126f ? 0x1p64f : 1.f;
    x.w[k] = x.w[k] * keep - (x.m[k] * __builtin_amdgcn_rcpf(den * up)) * up * rate;
  }
  if (WIDE) {
    if (it.w) store4(it.w, false, at, x.w);
    store4(it.p, it.p_bf16, at, x.w);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < left) {
        if (it.w) it.w[at + k] = x.w[k];
        if (it.p_bf16) Store<bf16_t>::store(it.p, at + k, x.w[k]); else Store<float>::store(it.p, at + k, x.w[k]);
      }
  }
  if (EIGHT) {
    // (the product is as good a scale as the quotient by 448, whose last bit differs for every second maximum: codes are worked out from the scale that is kept)
    const float new_ms = wave_most(fmaxf(fmaxf(fabsf(x.m[0]), fabsf(x.m[1])), fmaxf(fabsf(x.m[2]), fabsf(x.m[3])))) * (1.f / kTop8);
    const float new_vs = wave_most(fmaxf(fmaxf(root[0], root[1]), fmaxf(root[2], root[3]))) * (1.f / kTop8);
    const unsigned cm = pack8(x.m, unit_of(new_ms));
    unsigned cv = pack8(root, unit_of(new_vs));
    // a positive root never becomes 0: code 1, 2^-9, is the smallest
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if ((cv >> (8 * k) & 255u) == 0u && root[k] > 0.f) cv |= 1u << (8 * k);
    if (WIDE) {
      __builtin_nontemporal_store(cm, (unsigned*)((uint8_t*)it.m + at));
      __builtin_nontemporal_store(cv, (unsigned*)((uint8_t*)it.v + at));
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < left) {
          ((uint8_t*)it.m)[at + k] = (uint8_t)(cm >> (8 * k));
          ((uint8_t*)it.v)[at + k] = (uint8_t)(cv >> (8 * k));
        }
    }
    if (lane == 0) { it.ms[block] = new_ms; it.vs[block] = new_vs; }
  } else if (WIDE) {
    store4(it.m, false, at, x.m);
    store4(it.v, false, at, x.v);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < left) {
        ((float*)it.m)[at + k] = x.m[k];
        ((float*)it.v)[at + k] = x.v[k];
      }
  }
}

// Bound by memory: 133 M elements, 30 bytes each, in 665 us (6.0 TB/s), in 8 bits 18 bytes in 393.
// A wavefront takes 256 elements of a tensor, a block of the 8-bit states.  (Four blocks a wavefront, all of them asked for before the first is worked on:
// 133 M weights with the norm 865 us, in 8 bits 583; one, before the loads passed the caches, 847 and 554, since more wavefronts fit a compute unit and their phases overlap.)
template <bool EIGHT>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a) {
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  if (gs - gs != 0.f) return;                                             // NaN or infinite: the step is passed over
  const int i = find(a.first, a.count, blockIdx.x);
  const Item it = a.get(i);
  const double lr = a.lr_dev ? (double)*a.lr_dev : a.lr;
  float rate = a.rate, inv_root2 = a.inv_root2;
  if (a.lr_dev || a.step_dev) corrections(lr, a.beta1, a.beta2, a.step_dev ? max(*a.step_dev, 1) : a.step, rate, inv_root2);
  const float keep = (float)(1.0 - lr * it.decay);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long block = (long)(blockIdx.x - a.first[i]) * (kTile / kBlock) + wave, n = it.n;
  if (block * kBlock >= n) return;
  Block<EIGHT> x;
  if (it.wide && (block + 1) * kBlock <= n) {
    fetch<EIGHT, true>(x, it, block, lane);
    update<EIGHT, true>(x, it, a, block, lane, gs, keep, rate, inv_root2);
  } else {
    fetch<EIGHT, false>(x, it, block, lane);
    update<EIGHT, false>(x, it, a, block, lane, gs, keep, rate, inv_root2);
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
  // tensors of more elements than an item has are cut into pieces of whole tiles
  NormArgs a;
  a.part = part; a.count = 0;
  unsigned first = 0;
  long elements = 0;
  uint64_t bytes = 0;
  for (int i = 0; i < count; ++i) {
    elements += items[i].count;
    bytes += (uint64_t)items[i].count * (items[i].grad_dtype == LSTM_BF16_F32STATE ? 2 : 4);
  }
  const bool stream_past = bytes > kLastLevelBytes;
  const auto flush = [&] {
    if (a.count > 0) hipLaunchKernelGGL(stream_past ? grad_norm_kernel<true> : grad_norm_kernel<false>, dim3(first), dim3(256), 0, s, a);
    a.part += first;
    a.count = 0; first = 0;
  };
  const bool few = elements <= kNormFew && count <= kNormItems;
  for (int i = 0; i < count; ++i)
    for (long at = 0; at < items[i].count; at += kNormMost) {
      if (a.count == kNormItems || first >= (1u << 22)) flush();
      const bool bf16 = items[i].grad_dtype == LSTM_BF16_F32STATE;
      const long n = std::min((long)items[i].count - at, kNormMost);
      a.g[a.count] = (uint64_t)(uintptr_t)items[i].grad + (uint64_t)at * (bf16 ? 2 : 4) + (bf16 ? 1 : 0);
      a.n[a.count] = (unsigned)n; a.first[a.count++] = first;
      first += (unsigned)(few ? (n + kNormFewTile - 1) / kNormFewTile : (n + kNormTile - 1) / kNormTile);
    }
  if (few) {
    hipLaunchKernelGGL(grad_norm_few_kernel, dim3(1), dim3(1024), 0, s, a, first, max_norm, out);
    return hipGetLastError() == hipSuccess ? LSTM_OK : LSTM_ERR_HIP;
  }
  flush();
  hipLaunchKernelGGL(grad_norm_sum_kernel, dim3(1), dim3(1024), 0, s, part, (long)groups, max_norm, out);
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
  a.b1 = (float)d->beta1; a.nb1 = (float)(1.0 - d->beta1); a.b2 = (float)d->beta2; a.nb2 = (float)(1.0 - d->beta2);
  a.eps = d->eps > 0.0 ? std::max((float)d->eps, 0x1p-149f) : 0.f;           // (a positive eps stays positive)
  a.lr_dev = d->lr_dev; a.step_dev = d->step_dev; a.grad_scale = d->grad_scale;
  a.rate = a.inv_root2 = 1.f;
  if (!a.lr_dev && !a.step_dev) corrections(a.lr, a.beta1, a.beta2, a.step, a.rate, a.inv_root2);
  unsigned first = 0;
  const auto flush = [&] {
    if (a.count > 0) hipLaunchKernelGGL(eight ? adamw_kernel<true> : adamw_kernel<false>, dim3(first), dim3(256), 0, (hipStream_t)stream, a);
    a.count = 0; first = 0;
  };
  for (int i = 0; i < count; ++i)
    for (long at = 0; at < items[i].count; at += kMost) {
      if (a.count == kItems || first >= (1u << 22)) flush();
      const lstm_adamw_item& it = items[i];
      const bool pb = it.param_dtype == LSTM_BF16_F32STATE, gb = it.grad_dtype == LSTM_BF16_F32STATE;
      const long n = std::min((long)it.count - at, kMost), ss = at * (eight ? 1 : 4);
      const bool wide = (((uintptr_t)it.param & (pb ? 7 : 15)) | ((uintptr_t)it.grad & (gb ? 7 : 15)) | ((uintptr_t)it.master & 15) |
                         (((uintptr_t)it.m | (uintptr_t)it.v) & (eight ? 3 : 15))) == 0;
      const Item x = {(char*)it.param + at * (pb ? 2 : 4), it.master ? it.master + at : nullptr, (const char*)it.grad + at * (gb ? 2 : 4),
                      (char*)it.m + ss, (char*)it.v + ss, eight ? it.m_scale + at / kBlock : nullptr, eight ? it.v_scale + at / kBlock : nullptr,
                      (unsigned)n, pb, gb, wide, it.weight_decay};
      a.put(a.count++, x, first);
      first += (unsigned)((n + kTile - 1) / kTile);
    }
  flush();
  return hipGetLastError() == hipSuccess ? LSTM_OK : LSTM_ERR_HIP;
}

}  // extern "C"
