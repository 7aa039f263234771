// What becomes of a step's gradients: their global norm with the clip coefficient, and the AdamW update of many tensors in
// one launch, with moments in 32 bits or as 8-bit codes.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p -= lr (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + wd p)
//
// A handful of operations on every element read: memory bounds the large calls, launches the small ones.  The tensors'
// addresses travel as kernel arguments (no table in device memory: nothing to copy, and a captured launch carries its own).
#include "../../include/mrl.h"
#include "mrl_internal.h"
#include "mrl_vec.h"

#include <algorithm>
#include <cmath>
#include <new>

namespace mrl {
namespace {

constexpr int kNormChunk = 2048;             // elements of a tensor that a workgroup takes at a time: norm, eight a thread
constexpr int kAdamThreads = 64, kAdamChunk = kAdamThreads * 4;    // ... update, a wave and four a lane
constexpr int kStateBlock = kAdamChunk;      // elements that share a scale of 8-bit states

// ------------------------------------------------------------------ global norm
constexpr int kNormTensors = 96;             // a launch: 1.9 KB of arguments
constexpr int kNormBlocks = 2048;            // workgroups of a launch at most, a partial sum each
struct NormTable {
  const void* grad[kNormTensors];
  int64_t n[kNormTensors];
  int32_t chunk0[kNormTensors];              // the launch's chunks before the tensor's own; behind the last tensor INT32_MAX
  uint32_t bf16[kNormTensors / 32];
  int32_t chunks;
  double* parts;
};

// Index of the tensor that the launch's chunk belongs to: how many of the (ascending) first chunks are not above it, less one.
template <int kMost> __device__ inline int tensor_of(const int32_t* chunk0, int chunk) {
  const int lane = threadIdx.x & 63;
  int below = 0;
#pragma unroll
  for (int k = 0; k < kMost; k += 64) {
    const bool in = k + lane < kMost && chunk0[k + lane < kMost ? k + lane : 0] <= chunk;
    below += __popcll(__ballot(in));
  }
  return __builtin_amdgcn_readfirstlane(below - 1);
}

__device__ inline double wave_sum_f64(double x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
  return x;
}
template <int kWaves> __device__ inline double block_sum_f64(double x, double* sh) {
  x = wave_sum_f64(x);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s += sh[w];
  return s;
}

// A partial sum of squares for each workgroup, which takes every gridDim.x-th chunk.  A chunk that is squared and added in fp64 (exact squares of float and
// bf16) costs less than its read: 233 M floats in 151 us, 6.2 TB/s; with 1024 and 4096 workgroups in place of 2048 163 and 154.  (A kernel that only reads 4 GiB reaches
// 5.3 - 6.3 TB/s with plain loads and 5.7 - 7.1 with streamed ones, by its number of workgroups.)  A tensor's last chunk loads element by element, behind branches: of
// 57 small tensors, whose 164 chunks hold 57 such, 4.3 us.
__global__ __launch_bounds__(256) void k_square_sums(NormTable a) {
  __shared__ double sh[4];
  double s = 0.0;
  for (int chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    const int i = tensor_of<kNormTensors>(a.chunk0, chunk);
    const int64_t at = (int64_t)(chunk - a.chunk0[i]) * kNormChunk;
    const int left = (int)min((int64_t)kNormChunk, a.n[i] - at), c = threadIdx.x * 8;
    float g[8];
    const bool bf16 = a.bf16[i >> 5] >> (i & 31) & 1;
    const uint16_t* g16 = static_cast<const uint16_t*>(a.grad[i]) + at + c;
    const float* g32 = static_cast<const float*>(a.grad[i]) + at + c;
    if (left == kNormChunk) {
      if (bf16) {
        const u32x4 w = load_any<2, u32x4>(g16);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = e & 1 ? bf16_high(w[e >> 1]) : bf16_low(w[e >> 1]);
      } else {
        const u32x4 w0 = load_any<4, u32x4>(g32), w1 = load_any<4, u32x4>(g32 + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = __uint_as_float(e < 4 ? w0[e & 3] : w1[e & 3]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = c + e >= left ? 0.f : bf16 ? bf16_low(g16[e]) : g32[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fma((double)g[e], (double)g[e], s);
  }
  s = block_sum_f64<4>(s, sh);
  if (threadIdx.x == 0) a.parts[blockIdx.x] = s;
}

// out[0] = norm, out[1] = min(1, max_norm / norm), or NaN where the norm is no number.
__global__ __launch_bounds__(1024) void k_norm_coef(const double* parts, int n, double max_norm, float* out) {
  __shared__ double sh[16];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 1024) s += parts[i];
  s = block_sum_f64<16>(s, sh);
  if (threadIdx.x != 0) return;
  const double norm = sqrt(s), ratio = max_norm / norm;
  out[0] = (float)norm;
  out[1] = s < (double)INFINITY ? (ratio < 1.0 ? (float)ratio : 1.f) : __builtin_nanf("");
}

// ------------------------------------------------------------------ AdamW
template <bool kCodes> struct AdamTensor;
template <> struct AdamTensor<false> {
  float* param; uint16_t* copy; const void* grad; void* m; void* v;
  int64_t n; float weight_decay; uint32_t place_bf16 /*twice the place in the call, plus 1 where the gradient is bf16*/;
};
template <> struct AdamTensor<true> {
  float* param; uint16_t* copy; const void* grad; void* m; void* v; float* m_scale; float* v_scale;
  int64_t n; float weight_decay; uint32_t place_bf16;
};
template <bool kCodes> struct AdamTable {
  static constexpr int kTensors = kCodes ? 48 : 64;     // a launch: 3.8 and 3.9 KB of arguments
  AdamTensor<kCodes> t[kTensors];
  int32_t chunk0[kTensors];                             // as above
  int32_t chunks, skip_nonfinite;
  float lr, inv_fix1, inv_root_fix2;                    // 1 / (1 - b1^t), 1 / sqrt(1 - b2^t)
  float b1, one_b1, b2, one_b2, eps;
  double beta1, beta2;
  int64_t step;
  uint64_t seed;
  const float* lr_dev; const int64_t* step_dev; const float* coef;
};

// b1^t by squaring.
__host__ __device__ inline double power(double b, int64_t t) {
  double r = 1.0;
  for (; t > 0; t >>= 1) {
    if (t & 1) r *= b;
    b *= b;
  }
  return r;
}

// Random bits of element i of a tensor: mix(lo(i) ^ mix(key + hi(i))), the key mixed of the seed, the step and the tensor's place.
// Two rounds of multiplication and shift: every bit of the argument moves every bit of the result.
__host__ __device__ inline uint32_t mix(uint32_t x) {
  x = (x ^ x >> 16) * 0x6A09E667u;           // (fractional bits of the square roots of 2 and 3)
  x = (x ^ x >> 15) * 0xBB67AE85u;
  return x ^ x >> 16;
}
__device__ inline uint32_t key_of(uint64_t seed, int64_t step, uint32_t place) {
  return mix((uint32_t)seed ^ mix((uint32_t)(seed >> 32) ^ mix((uint32_t)step ^ mix(place))));
}

// x >= 0, at most 448 (a little above by rounding): the e4m3 value below or above, above with the probability of the fraction.  u: 16
// random bits, a fraction of the step.
__device__ inline float to_code(float x, uint32_t u16) {
  const uint32_t top = __float_as_uint(x) & 0x7f800000u;
  const uint32_t binade = top > (121u << 23) ? top : 121u << 23;                                     // subnormals: that of 2^-6
  const float per_step = __uint_as_float((257u << 23) - binade), step = __uint_as_float(binade - (3u << 23));
  return fminf(floorf(fmaf((float)u16, 0x1p-16f, x * per_step)) * step, kE4m3Max);
}

// Products and sums that are rounded one by one: the compiler may not make a fused one of two.
__device__ inline float times(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}
__device__ inline float plus(float a, float b) {
#pragma clang fp contract(off)
  return a + b;
}

// The scale of a block with this largest magnitude.  x - x is zero, or NaN where x is infinite: under an infinite scale sqrt(v) would decode to infinity
// and hold the block's weights where they are for good.
__device__ inline float scale_or_nan(float x) { return plus(times(x, 1.f / kE4m3Max), plus(x, -x)); }

// What the elements of a launch share.
struct Rates { float lr, inv_fix1, inv_root_fix2, coef, b1, one_b1, b2, one_b2, eps, decay; };

// Four elements of a tensor and their moments, in registers.
struct Four {
  float p[4], g[4], m[4], v[4], root[4];
  __device__ void update(const Rates& r) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float ge = g[e] * r.coef;
      m[e] = plus(times(r.b1, m[e]), times(r.one_b1, ge));
      v[e] = plus(times(r.b2, v[e]), times(times(r.one_b2, ge), ge));
      root[e] = sqrtf(v[e]);
      p[e] = fmaf(-r.lr, fmaf(r.decay, p[e], m[e] * r.inv_fix1 / fmaf(root[e], r.inv_root_fix2, r.eps)), p[e]);
    }
  }
  // Codes of the moments and the block's scales; the wave's 64 fours are a block, elements from `some` on count as zeros.
  __device__ void encode(int some, uint32_t first, uint32_t key, uint32_t* mw, uint32_t* vw, float* m_scale, float* v_scale) {
    uint32_t m_most = kScaleLeast, v_most = kScaleLeast;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (e >= some) m[e] = root[e] = 0.f;
      m_most = larger(m_most, magnitude(m[e]));
      v_most = larger(v_most, magnitude(root[e]));
    }
    const float m_max = __uint_as_float(lanes_max<64>(m_most)), v_max = __uint_as_float(lanes_max<64>(v_most));
    const float m_inv = times(1.f / m_max, kE4m3Max), v_inv = times(1.f / v_max, kE4m3Max);
    float mq[4], vq[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t bits = mix((first + e) ^ key);
      mq[e] = copysignf(to_code(fabsf(m[e]) * m_inv, bits & 0xffffu), m[e]);
      // a positive root keeps a positive code: at zero the next step would divide by that step's gradient alone
      vq[e] = fmaxf(to_code(root[e] * v_inv, bits >> 16), root[e] > 0.f ? 0x1p-9f : 0.f);
    }
    *mw = pack_e4m3(mq[0], mq[1], mq[2], mq[3]);
    *vw = pack_e4m3(vq[0], vq[1], vq[2], vq[3]);
    *m_scale = scale_or_nan(m_max);
    *v_scale = scale_or_nan(v_max);
  }
  __device__ void decode(uint32_t mw, uint32_t vw, float m_scale, float v_scale) {
    const auto m01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mw, false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mw, true);
    const auto v01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)vw, false), v23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)vw, true);
    m[0] = times(m01[0], m_scale); m[1] = times(m01[1], m_scale); m[2] = times(m23[0], m_scale); m[3] = times(m23[1], m_scale);
    v[0] = times(v01[0], v_scale); v[1] = times(v01[1], v_scale); v[2] = times(v23[0], v_scale); v[3] = times(v23[1], v_scale);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = times(v[e], v[e]);
  }
};
__device__ inline u32x4 as_words(const float (&x)[4]) {
  return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}
__device__ inline void as_floats(u32x4 w, float (&x)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(w[e]);
}

// A workgroup of one wave takes 256 elements of a tensor, which are a block of 8-bit states.  Memory bounds it: 30 bytes an element with 32-bit moments
// (233 M in 1140 - 1180 us from card to card, 5.9 - 6.1 TB/s), 18 with 8-bit ones (263 M in 755 - 805 us, 5.9 - 6.3 TB/s), where the hash, the roots and the quotients fit beside
// the loads.  With the step on the device each wave computes its two corrections before its first load: 32-bit moments take no longer (1154), 8-bit ones 919 - 986.  Everything passes
// the caches: nothing is read again before all the rest has gone through them (kept 1315 us, loads or stores streamed 1303 and 1311, both 1252, then in
// workgroups of one wave and 256 elements 1161; of 128, 512 and 1024 threads 1182, 1249, 1230).
template <bool kCodes>
__global__ __launch_bounds__(kAdamThreads) void k_adamw(AdamTable<kCodes> a) {
  const int chunk = (int)(blockIdx.y * gridDim.x + blockIdx.x);       // (at most 2^30 and the rest of a row of workgroups)
  if (chunk >= a.chunks) return;
  const int i = tensor_of<AdamTable<kCodes>::kTensors>(a.chunk0, chunk);
  const AdamTensor<kCodes>& t = a.t[i];
  const bool grad_bf16 = t.place_bf16 & 1;
  const int64_t at = (int64_t)(chunk - a.chunk0[i]) * kAdamChunk;
  Rates r = {a.lr, a.inv_fix1, a.inv_root_fix2, a.coef != nullptr ? *a.coef : 1.f, a.b1, a.one_b1, a.b2, a.one_b2, a.eps, t.weight_decay};
  if (a.skip_nonfinite && !(fabsf(r.coef) < INFINITY)) return;
  int64_t step = a.step;
  if (a.lr_dev != nullptr) r.lr = *a.lr_dev;
  if (a.step_dev != nullptr) {
    step = max(*a.step_dev, (int64_t)1);
    r.inv_fix1 = (float)(1.0 / (1.0 - power(a.beta1, step)));
    r.inv_root_fix2 = (float)(1.0 / sqrt(1.0 - power(a.beta2, step)));
  }
  const int lane = threadIdx.x, c = lane * 4;
  const int left = (int)min((int64_t)kAdamChunk, t.n - at);
  const uint32_t key = kCodes ? mix(key_of(a.seed, step, t.place_bf16 >> 1) + (uint32_t)(at >> 32)) : 0;
  float* const param = t.param + at;
  uint16_t* const copy = t.copy + at;
  const float* const grad = static_cast<const float*>(t.grad) + at;
  const uint16_t* const grad16 = static_cast<const uint16_t*>(t.grad) + at;
  float *const m = static_cast<float*>(t.m) + at, *const v = static_cast<float*>(t.v) + at;
  uint8_t *const mc = static_cast<uint8_t*>(t.m) + at, *const vc = static_cast<uint8_t*>(t.v) + at;
  float *m_scale = nullptr, *v_scale = nullptr;
  if constexpr (kCodes) { m_scale = t.m_scale + at / kStateBlock; v_scale = t.v_scale + at / kStateBlock; }
  if (left == kAdamChunk) {
    Four f;
    const u32x4 pw = load_stream<4, u32x4>(param + c);
    if constexpr (kCodes) {
      const uint32_t mw = load_stream<1, uint32_t>(mc + c), vw = load_stream<1, uint32_t>(vc + c);
      f.decode(mw, vw, *m_scale, *v_scale);
    } else {
      const u32x4 mw = load_stream<4, u32x4>(m + c), vw = load_stream<4, u32x4>(v + c);
      as_floats(mw, f.m);
      as_floats(vw, f.v);
    }
    if (grad_bf16) {
      const u32x2 w = load_stream<2, u32x2>(grad16 + c);
      as_floats(u32x4{w[0] << 16, w[0] & 0xffff0000u, w[1] << 16, w[1] & 0xffff0000u}, f.g);
    } else {
      as_floats(load_stream<4, u32x4>(grad + c), f.g);
    }
    as_floats(pw, f.p);
    f.update(r);
    store_stream<4>(param + c, as_words(f.p));
    if (t.copy != nullptr) store_stream<2>(copy + c, u32x2{pack_bf16(f.p[0], f.p[1]), pack_bf16(f.p[2], f.p[3])});
    if constexpr (kCodes) {
      uint32_t mw, vw;
      float ms, vs;
      f.encode(4, (uint32_t)(at + c), key, &mw, &vw, &ms, &vs);
      store_stream<1>(mc + c, mw);
      store_stream<1>(vc + c, vw);
      if (lane == 0) { *m_scale = ms; *v_scale = vs; }
    } else {
      store_stream<4>(m + c, as_words(f.m));
      store_stream<4>(v + c, as_words(f.v));
    }
    return;
  }
  // a tensor's last chunk, element by element
  const int some = min(max(left - c, 0), 4);
  Four f;
  uint32_t mw = 0, vw = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool in = e < some;
    f.p[e] = in ? param[c + e] : 0.f;
    f.g[e] = !in ? 0.f : grad_bf16 ? bf16_low(grad16[c + e]) : grad[c + e];
    if constexpr (kCodes) {
      if (in) { mw |= (uint32_t)mc[c + e] << 8 * e; vw |= (uint32_t)vc[c + e] << 8 * e; }
    } else {
      f.m[e] = in ? m[c + e] : 0.f;
      f.v[e] = in ? v[c + e] : 0.f;
    }
  }
  if constexpr (kCodes) f.decode(mw, vw, *m_scale, *v_scale);
  f.update(r);
  float ms, vs;
  if constexpr (kCodes) f.encode(some, (uint32_t)(at + c), key, &mw, &vw, &ms, &vs);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (e >= some) continue;
    param[c + e] = f.p[e];
    if (t.copy != nullptr) copy[c + e] = (uint16_t)pack_bf16(f.p[e], 0.f);
    if constexpr (kCodes) {
      mc[c + e] = (uint8_t)(mw >> 8 * e);
      vc[c + e] = (uint8_t)(vw >> 8 * e);
    } else {
      m[c + e] = f.m[e];
      v[c + e] = f.v[e];
    }
  }
  if constexpr (kCodes) {
    if (lane == 0) { *m_scale = ms; *v_scale = vs; }
  }
}

// ------------------------------------------------------------------ host
constexpr int64_t kMostWide = 1 << 25;
constexpr int64_t kMaxElements = (int64_t)1 << 40;
int64_t chunks_of(int64_t n, int chunk) { return (n + chunk - 1) / chunk; }

int check_tensors(const mrl_param_tensor* t, int32_t count, bool update, bool codes) {
  if (count < 0) return MRL_ERR_SHAPE;
  if (count > 0 && t == nullptr) return MRL_ERR_NULL;
  int64_t chunks = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (t[i].n < 0 || t[i].n > kMaxElements) return MRL_ERR_SHAPE;
    if (t[i].grad_dtype != MRL_F32 && t[i].grad_dtype != MRL_BF16) return MRL_ERR_DTYPE;
    if (t[i].n == 0) continue;
    chunks += chunks_of(t[i].n, update ? kAdamChunk : kNormChunk);
    if (!t[i].grad) return MRL_ERR_NULL;
    if (!update) continue;
    if (!t[i].param || !t[i].m || !t[i].v || (codes && (!t[i].m_scale || !t[i].v_scale))) return MRL_ERR_NULL;
    if (!(t[i].weight_decay >= 0.f && t[i].weight_decay < INFINITY)) return MRL_ERR_CONFIG;
  }
  return chunks <= (int64_t)1 << 30 ? MRL_OK : MRL_ERR_SHAPE;            // (256 elements each: more than a device holds)
}

// Calls f(first, last) for the tensors of each launch: at most kMost of them that are not empty.
template <int kMost, class F> void in_launches(const mrl_param_tensor* t, int32_t count, F f) {
  int32_t first = 0, held = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (t[i].n == 0) continue;
    if (held == kMost) { f(first, i); first = i; held = 0; }
    ++held;
  }
  if (held > 0) f(first, count);
}

// A partial sum for each workgroup of each launch.
size_t norm_bytes(const mrl_param_tensor* t, int32_t count) {
  int64_t parts = 0;
  in_launches<kNormTensors>(t, count, [&](int32_t first, int32_t last) {
    int64_t chunks = 0;
    for (int32_t i = first; i < last; ++i) chunks += chunks_of(t[i].n, kNormChunk);
    parts += std::min<int64_t>(chunks, kNormBlocks);
  });
  return (size_t)round_up(parts * 8 + 8, 256);
}

template <bool kCodes>
void go_adamw(const mrl_param_tensor* tensors, int32_t count, const mrl_adamw_config& cfg, const float* grad_coef, hipStream_t s) {
  using Table = AdamTable<kCodes>;
  static_assert(sizeof(Table) <= 4096, "kernel arguments");
  in_launches<Table::kTensors>(tensors, count, [&](int32_t first, int32_t last) {
    Table a = {};
    int k = 0;
    int64_t chunks = 0;
    for (int32_t i = first; i < last; ++i) {
      const mrl_param_tensor& t = tensors[i];
      if (t.n == 0) continue;
      AdamTensor<kCodes>& to = a.t[k];
      to.param = t.param; to.copy = static_cast<uint16_t*>(t.copy); to.grad = t.grad; to.m = t.m; to.v = t.v;
      if constexpr (kCodes) { to.m_scale = t.m_scale; to.v_scale = t.v_scale; }
      to.n = t.n; to.weight_decay = t.weight_decay; to.place_bf16 = 2u * (uint32_t)i + (t.grad_dtype == MRL_BF16);
      a.chunk0[k] = (int32_t)chunks;
      chunks += chunks_of(t.n, kAdamChunk);
      ++k;
    }
    for (; k < Table::kTensors; ++k) a.chunk0[k] = INT32_MAX;
    a.skip_nonfinite = cfg.skip_nonfinite;
    a.beta1 = cfg.beta1; a.beta2 = cfg.beta2;
    a.lr = (float)cfg.lr;
    a.b1 = (float)cfg.beta1; a.one_b1 = (float)(1.0 - cfg.beta1);
    a.b2 = (float)cfg.beta2; a.one_b2 = (float)(1.0 - cfg.beta2);
    a.eps = (float)cfg.eps;
    a.step = cfg.step; a.seed = cfg.seed;
    a.inv_fix1 = (float)(1.0 / (1.0 - power(cfg.beta1, cfg.step)));
    a.inv_root_fix2 = (float)(1.0 / std::sqrt(1.0 - power(cfg.beta2, cfg.step)));
    a.lr_dev = cfg.lr_dev; a.step_dev = cfg.step_dev; a.coef = grad_coef;
    a.chunks = (int32_t)chunks;
    // (a launch has fewer than 2^32 threads along x)
    const int64_t wide = std::min<int64_t>(chunks, kMostWide);
    hipLaunchKernelGGL(k_adamw<kCodes>, dim3((unsigned)wide, (unsigned)((chunks + wide - 1) / wide)), dim3(kAdamThreads), 0, s, a);
  });
}

}  // namespace
}  // namespace mrl

using namespace mrl;

extern "C" size_t mrl_grad_norm_workspace(const mrl_param_tensor* tensors, int32_t count) {
  if (check_tensors(tensors, count, false, false) != MRL_OK) return 0;
  return norm_bytes(tensors, count);
}

extern "C" int mrl_grad_norm(const mrl_param_tensor* tensors, int32_t count, double max_norm, float* out_norm_coef, void* workspace,
                             size_t workspace_bytes, void* stream) {
  int rc = check_tensors(tensors, count, false, false);
  if (rc != MRL_OK) return rc;
  if (!out_norm_coef) return MRL_ERR_NULL;
  if (!(max_norm > 0.0)) return MRL_ERR_CONFIG;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < norm_bytes(tensors, count)) return MRL_ERR_WORKSPACE;
  rc = require_gfx950();
  if (rc != MRL_OK) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  double* const parts = static_cast<double*>(workspace);
  int n_parts = 0;
  in_launches<kNormTensors>(tensors, count, [&](int32_t first, int32_t last) {
    NormTable a = {};
    int k = 0;
    int64_t chunks = 0;
    for (int32_t i = first; i < last; ++i) {
      if (tensors[i].n == 0) continue;
      a.grad[k] = tensors[i].grad;
      a.n[k] = tensors[i].n;
      a.chunk0[k] = (int32_t)chunks;
      if (tensors[i].grad_dtype == MRL_BF16) a.bf16[k >> 5] |= 1u << (k & 31);
      chunks += chunks_of(tensors[i].n, kNormChunk);
      ++k;
    }
    for (; k < kNormTensors; ++k) a.chunk0[k] = INT32_MAX;
    a.chunks = (int32_t)chunks;
    a.parts = parts + n_parts;
    const int blocks = (int)std::min<int64_t>(chunks, kNormBlocks);
    n_parts += blocks;
    hipLaunchKernelGGL(k_square_sums, dim3(blocks), dim3(256), 0, s, a);
  });
  hipLaunchKernelGGL(k_norm_coef, dim3(1), dim3(1024), 0, s, parts, n_parts, max_norm, out_norm_coef);
  return hipGetLastError() == hipSuccess ? MRL_OK : MRL_ERR_DEVICE;
}

extern "C" int mrl_adamw(const mrl_param_tensor* tensors, int32_t count, const mrl_adamw_config* cfg, const float* grad_coef, void* stream) {
  if (!cfg) return MRL_ERR_NULL;
  if (cfg->state_dtype != MRL_F32 && cfg->state_dtype != MRL_E4M3) return MRL_ERR_DTYPE;
  const bool codes = cfg->state_dtype == MRL_E4M3;
  int rc = check_tensors(tensors, count, true, codes);
  if (rc != MRL_OK) return rc;
  if (!(cfg->lr >= 0.0 && cfg->lr < 1e30) || !(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0) ||
      !(cfg->eps >= 1e-30 && cfg->eps < 1e30) || (cfg->step_dev == nullptr && cfg->step < 1) || (cfg->skip_nonfinite != 0 && cfg->skip_nonfinite != 1))
    return MRL_ERR_CONFIG;
  if (count == 0) return MRL_OK;
  rc = require_gfx950();
  if (rc != MRL_OK) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (codes) go_adamw<true>(tensors, count, *cfg, grad_coef, s);
  else go_adamw<false>(tensors, count, *cfg, grad_coef, s);
  return hipGetLastError() == hipSuccess ? MRL_OK : MRL_ERR_DEVICE;
}

extern "C" int mrl_adamw_check(const mrl_param_tensor* tensors, int32_t count, int32_t state_dtype) {
  if (state_dtype != MRL_F32 && state_dtype != MRL_E4M3) return MRL_ERR_DTYPE;
  const bool codes = state_dtype == MRL_E4M3;
  const int rc = check_tensors(tensors, count, true, codes);
  if (rc != MRL_OK || count == 0) return rc;
  struct Range { uintptr_t first, last; bool written; };
  const size_t most = (size_t)count * 7;
  Range* const r = new (std::nothrow) Range[most];
  if (r == nullptr) return MRL_ERR_DEVICE;
  size_t k = 0;
  auto add = [&](const void* p, int64_t bytes, bool written) {
    if (p != nullptr && bytes > 0) r[k++] = {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes, written};
  };
  for (int32_t i = 0; i < count; ++i) {
    const mrl_param_tensor& t = tensors[i];
    const int64_t moment = codes ? 1 : 4, scales = codes ? (t.n + kStateBlock - 1) / kStateBlock * 4 : 0;
    add(t.param, t.n * 4, true);
    add(t.copy, t.n * 2, true);
    add(t.m, t.n * moment, true);
    add(t.v, t.n * moment, true);
    add(t.m_scale, scales, true);
    add(t.v_scale, scales, true);
    add(t.grad, t.n * (t.grad_dtype == MRL_BF16 ? 2 : 4), false);
  }
  std::sort(r, r + k, [](const Range& a, const Range& b) { return a.first < b.first; });
  // (two gradients may overlap: nothing writes them)
  uintptr_t written_to = 0, read_to = 0;
  bool apart = true;
  for (size_t i = 0; i < k && apart; ++i) {
    apart = r[i].first >= written_to && !(r[i].written && r[i].first < read_to);
    uintptr_t& to = r[i].written ? written_to : read_to;
    to = std::max(to, r[i].last);
  }
  delete[] r;
  return apart ? MRL_OK : MRL_ERR_CONFIG;
}
