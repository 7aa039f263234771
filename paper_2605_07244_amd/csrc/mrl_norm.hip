// Root-mean-square norm of hidden states, with the residual's addition and outputs in 32, 16 or 8 bits, and its backward
// pass.  Row n of [N, d]:
//   h = x + residual,  r = 1 / sqrt(mean h^2 + eps),  y = h r w;     8 bits: y ~ scale q, scale = max |y| / 448
//   g = dy w,  u = h r,  dx = r (g - u mean(g u)) + d_residual,  dw = sum over rows of dy u
// Both read and write every element once and do a dozen operations on it: memory bounds them.  A row stays in registers
// between its sum and its output.
#include "../../include/mrl.h"
#include "mrl_internal.h"
#include "mrl_vec.h"

namespace mrl {
namespace {

struct NormArgs {
  const void* x; const void* residual; const void* w; const uint8_t* mask;
  int64_t N; int d; float eps;
  int w_bf16, y_type /*mrl_dtype*/, scale_block;
  void* sum; void* y; float* scale;
};

// Sum (or maximum) over the kT threads that share a row; `sh`: a slot per wave, used by nothing else between two barriers.
template <int kT> __device__ inline float group_sum(float x, float* sh) {
  x = wave_sum_f32(x);
  if (kT == 64) return x;
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < kT / 64; ++w) s += sh[w];
  return s;
}
template <int kT> __device__ inline uint32_t group_max(uint32_t x, uint32_t* sh) {
  x = wave_max(x);
  if (kT == 64) return x;
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  uint32_t m = 0;
#pragma unroll
  for (int w = 0; w < kT / 64; ++w) m = larger(m, sh[w]);
  return m;
}

__device__ inline void load_weights(const void* w, bool bf16, int c, int d, float (&out)[8]) {
  if (bf16) {
    Eight<true> v;
    v.load(w, c, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = v[e];
  } else {
    Eight<false> v;
    v.load(w, c, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = v[e];
  }
}

// kT threads take a row, each kNV times eight elements, kT * 8 apart.  kRes: 0 no residual, 1 bf16, 2 float.
template <bool kXBf16, int kRes, int kT, int kNV>
__global__ __launch_bounds__(kT < 256 ? 256 : kT) void k_rms_norm(NormArgs a) {
  __shared__ float sh_sum[16];
  __shared__ uint32_t sh_max[16];
  constexpr int kRows = kT < 256 ? 256 / kT : 1;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kT;
  if (row >= a.N) return;                               // (whole waves; with more waves a row there is one row a block)
  const int t = threadIdx.x % kT, d = a.d;
  const int scales = a.scale_block ? (d + 127) / 128 : 1;
  const char* x = static_cast<const char*>(a.x) + row * d * (kXBf16 ? 2 : 4);
  const char* res = static_cast<const char*>(a.residual) + row * d * (kRes == 1 ? 2 : 4);
  char* sum = static_cast<char*>(a.sum) + row * d * (kRes == 1 ? 2 : 4);
  char* y = static_cast<char*>(a.y) + row * d * (a.y_type == MRL_F32 ? 4 : a.y_type == MRL_BF16 ? 2 : 1);
  float h[kNV][8];
  const bool scored = a.mask == nullptr || a.mask[row] != 0;
  if (scored) {
    Eight<kXBf16> xv[kNV];
    Eight<kRes == 1> rv[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      const int c = (i * kT + t) * 8;
      xv[i].load(x, c, d);
      if (kRes) rv[i].load(res, c, d);
    }
#pragma unroll
    for (int i = 0; i < kNV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] = kRes ? xv[i][e] + rv[i][e] : xv[i][e];
  } else {
#pragma unroll
    for (int i = 0; i < kNV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] = 0.f;
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kNV; ++i) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(h[i][e], h[i][e], s);
    if (kRes) store_eight(sum, kRes == 1, (i * kT + t) * 8, d, h[i]);
  }
  s = group_sum<kT>(s, sh_sum);
  const float r = 1.f / sqrtf(s / (float)d + a.eps);
#pragma unroll
  for (int i = 0; i < kNV; ++i) {
    float w[8];
    load_weights(a.w, a.w_bf16, (i * kT + t) * 8, d, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[i][e] = scored ? h[i][e] * r * w[e] : 0.f;
  }
  if (a.y_type != MRL_E4M3) {
#pragma unroll
    for (int i = 0; i < kNV; ++i) store_eight(y, a.y_type == MRL_BF16, (i * kT + t) * 8, d, h[i]);
    return;
  }
  uint32_t most[kNV];
#pragma unroll
  for (int i = 0; i < kNV; ++i) {
    most[i] = kScaleLeast;
#pragma unroll
    for (int e = 0; e < 8; ++e) most[i] = larger(most[i], magnitude(h[i][e]));
  }
  if (a.scale_block) {                                  // 128 columns are 16 lanes
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      most[i] = row16_max(most[i]);
      const int block = (i * kT + t) / 16;
      if ((t & 15) == 0 && block < scales) a.scale[row * scales + block] = __uint_as_float(most[i]) / kE4m3Max;
    }
  } else {
#pragma unroll
    for (int i = 1; i < kNV; ++i) most[0] = larger(most[0], most[i]);
    most[0] = group_max<kT>(most[0], sh_max);
#pragma unroll
    for (int i = 1; i < kNV; ++i) most[i] = most[0];
    if (t == 0) a.scale[row] = __uint_as_float(most[0]) / kE4m3Max;
  }
#pragma unroll
  for (int i = 0; i < kNV; ++i) {
    const float inverse = kE4m3Max / __uint_as_float(most[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[i][e] *= inverse;
    store_eight_e4m3(y, (i * kT + t) * 8, d, h[i]);
  }
}

struct NormBackArgs {
  const void* dy; const void* h; const void* w; const void* d_residual; const uint8_t* mask;
  int64_t N; int d; float eps;
  int w_bf16, dx_bf16;
  void* dx; float* parts /*[gridDim.x][ld] | nullptr*/; int ld;
};

// Rows of a workgroup one after the other (kT < 256: 256 / kT of them side by side); the columns' sums of dy u stay in registers until the last row,
// then the rows that were side by side are added in LDS, in their order, and the workgroup writes one row of partial sums.
template <bool kHBf16, bool kDyBf16, int kT, int kNV>
__global__ __launch_bounds__(kT < 256 ? 256 : kT) void k_rms_norm_back(NormBackArgs a) {
  extern __shared__ float lds[];                        // kT < 256: [d] sums; else two sets of two sums a wave
  constexpr int kRows = kT < 256 ? 256 / kT : 1;
  const int t = threadIdx.x % kT, side = threadIdx.x / kT, d = a.d;
  float acc[kNV][8], w[kNV][8];                         // (weights stay in registers, too: every row needs them twice)
#pragma unroll
  for (int i = 0; i < kNV; ++i) {
    load_weights(a.w, a.w_bf16, (i * kT + t) * 8, d, w[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[i][e] = 0.f;
  }
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * kRows + side; row < a.N; row += (int64_t)gridDim.x * kRows) {
    const char* res = static_cast<const char*>(a.d_residual) + row * d * (kHBf16 ? 2 : 4);
    char* dx = static_cast<char*>(a.dx) + row * d * (a.dx_bf16 ? 2 : 4);
    Eight<kHBf16> hv[kNV], rv[kNV];
    Eight<kDyBf16> gv[kNV];
    const bool scored = a.mask == nullptr || a.mask[row] != 0;
    if (a.d_residual != nullptr) {
#pragma unroll
      for (int i = 0; i < kNV; ++i) rv[i].load(res, (i * kT + t) * 8, d);
    }
    if (!scored) {
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        float out[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = a.d_residual != nullptr ? rv[i][e] : 0.f;
        store_eight(dx, a.dx_bf16, (i * kT + t) * 8, d, out);
      }
      continue;
    }
    const char* h = static_cast<const char*>(a.h) + row * d * (kHBf16 ? 2 : 4);
    const char* dy = static_cast<const char*>(a.dy) + row * d * (kDyBf16 ? 2 : 4);
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      hv[i].load(h, (i * kT + t) * 8, d);
      gv[i].load(dy, (i * kT + t) * 8, d);
    }
    float hh = 0.f, gh = 0.f;
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        hh = fmaf(hv[i][e], hv[i][e], hh);
        gh = fmaf(gv[i][e] * w[i][e], hv[i][e], gh);
      }
    }
    hh = wave_sum_f32(hh);
    gh = wave_sum_f32(gh);
    if (kT > 64) {                                      // (two sets of slots in turn: one barrier a row)
      float* sh = lds + turn * 32;
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) { sh[threadIdx.x >> 6] = hh; sh[16 + (threadIdx.x >> 6)] = gh; }
      __syncthreads();
      hh = gh = 0.f;
#pragma unroll
      for (int w = 0; w < kT / 64; ++w) { hh += sh[w]; gh += sh[16 + w]; }
    }
    const float r = 1.f / sqrtf(hh / (float)d + a.eps), along = gh * r / (float)d;
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      float out[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float u = hv[i][e] * r;
        acc[i][e] = fmaf(gv[i][e], u, acc[i][e]);
        out[e] = r * (gv[i][e] * w[i][e] - u * along);
        if (a.d_residual != nullptr) out[e] += rv[i][e];
      }
      store_eight(dx, a.dx_bf16, (i * kT + t) * 8, d, out);
    }
  }
  if (a.parts == nullptr) return;
  float* part = a.parts + (int64_t)blockIdx.x * a.ld;
  if (kRows > 1) {
    for (int s = 0; s < kRows; ++s) {
      if (side == s) {
#pragma unroll
        for (int i = 0; i < kNV; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int c = (i * kT + t) * 8 + e;
            if (c >= d) continue;
            const float sum = s > 0 ? lds[c] + acc[i][e] : acc[i][e];
            if (s < kRows - 1) lds[c] = sum; else part[c] = sum;
          }
      }
      __syncthreads();
    }
  } else {
#pragma unroll
    for (int i = 0; i < kNV; ++i) store_eight(part, false, (i * kT + t) * 8, d, acc[i]);
  }
}

// dw[c] = (or +=) sum of the workgroups' partial sums, in fp64 in a fixed order: 16 columns a workgroup, 64 threads along the partials.
__global__ __launch_bounds__(256) void k_rms_norm_dw(const float* parts, int n_parts, int ld, int d, int accumulate, float* dw) {
  __shared__ double sh[4][16];
  const int c0 = blockIdx.x * 16 + (threadIdx.x & 3) * 4, lane = threadIdx.x & 63;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  if (c0 < ld) {
    for (int p = threadIdx.x >> 2; p < n_parts; p += 64) {
      const float4 v = *reinterpret_cast<const float4*>(parts + (int64_t)p * ld + c0);
      s[0] += (double)v.x; s[1] += (double)v.y; s[2] += (double)v.z; s[3] += (double)v.w;
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int off = 4; off < 64; off <<= 1) s[k] += __shfl_xor(s[k], off);
    if (lane < 4) sh[threadIdx.x >> 6][lane * 4 + k] = s[k];
  }
  __syncthreads();
  const int c = blockIdx.x * 16 + threadIdx.x;
  if (threadIdx.x < 16 && c < d) {
    double total = (sh[0][threadIdx.x] + sh[1][threadIdx.x]) + (sh[2][threadIdx.x] + sh[3][threadIdx.x]);
    if (accumulate) total += (double)dw[c];
    dw[c] = (float)total;
  }
}

constexpr int kMaxWidth = 16384;                         // 1024 threads, 16 elements each

// Threads that share a row, and how many times eight elements each takes.
struct Shape { int threads, vectors; };
Shape norm_shape(int64_t N, int d) {
  const int v = (d + 7) / 8;
  if (v <= 64) return {64, 1};
  if (N >= 1024 && v <= 512) return {64, v <= 128 ? 2 : v <= 256 ? 4 : 8};
  if (v <= 1024) return {256, v <= 256 ? 1 : v <= 512 ? 2 : 4};
  return {1024, 2};
}
Shape back_shape(int d) {
  const int v = (d + 7) / 8;
  if (v <= 128) return {64, v <= 64 ? 1 : 2};
  if (v <= 1024) return {256, v <= 256 ? 1 : v <= 512 ? 2 : 4};
  return {512, 4};
}
int rows_side_by_side(const Shape& s) { return s.threads < 256 ? 256 / s.threads : 1; }
int back_blocks(int64_t N, int d) {
  const int rows = rows_side_by_side(back_shape(d));
  const int64_t b = (N + rows - 1) / rows;
  return (int)(b < 1024 ? b : 1024);
}

template <bool kXBf16, int kRes> void go_norm(const NormArgs& a, hipStream_t s) {
  const Shape sh = norm_shape(a.N, a.d);
  const int rows = rows_side_by_side(sh);
  const dim3 grid((unsigned)((a.N + rows - 1) / rows)), block(sh.threads < 256 ? 256 : sh.threads);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
  if (sh.threads == 64) {
    if (sh.vectors == 1) go(k_rms_norm<kXBf16, kRes, 64, 1>);
    else if (sh.vectors == 2) go(k_rms_norm<kXBf16, kRes, 64, 2>);
    else if (sh.vectors == 4) go(k_rms_norm<kXBf16, kRes, 64, 4>);
    else go(k_rms_norm<kXBf16, kRes, 64, 8>);
  } else if (sh.threads == 256) {
    if (sh.vectors == 1) go(k_rms_norm<kXBf16, kRes, 256, 1>);
    else if (sh.vectors == 2) go(k_rms_norm<kXBf16, kRes, 256, 2>);
    else go(k_rms_norm<kXBf16, kRes, 256, 4>);
  } else {
    go(k_rms_norm<kXBf16, kRes, 1024, 2>);
  }
}

template <bool kHBf16, bool kDyBf16> void go_back(const NormBackArgs& a, hipStream_t s) {
  const Shape sh = back_shape(a.d);
  const dim3 grid((unsigned)back_blocks(a.N, a.d)), block(sh.threads < 256 ? 256 : sh.threads);
  const size_t lds = sh.threads < 256 ? (size_t)a.d * 4 : 64 * 4;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, lds, s, a); };
  if (sh.threads == 64) {
    if (sh.vectors == 1) go(k_rms_norm_back<kHBf16, kDyBf16, 64, 1>);
    else go(k_rms_norm_back<kHBf16, kDyBf16, 64, 2>);
  } else if (sh.threads == 256) {
    if (sh.vectors == 1) go(k_rms_norm_back<kHBf16, kDyBf16, 256, 1>);
    else if (sh.vectors == 2) go(k_rms_norm_back<kHBf16, kDyBf16, 256, 2>);
    else go(k_rms_norm_back<kHBf16, kDyBf16, 256, 4>);
  } else {
    go(k_rms_norm_back<kHBf16, kDyBf16, 512, 4>);
  }
}

bool is_float_type(int32_t t) { return t == MRL_F32 || t == MRL_BF16; }
constexpr int64_t kMaxRows = (int64_t)1 << 30;

}  // namespace
}  // namespace mrl

using namespace mrl;

extern "C" int mrl_rms_norm(const void* x, const void* residual, const void* weight, const uint8_t* token_mask, int64_t N, int32_t d,
                            float eps, int32_t x_dtype, int32_t residual_dtype, int32_t weight_dtype, int32_t y_dtype, int32_t scale_block,
                            void* out_sum, void* out_y, float* out_scale, void* stream) {
  if (N < 0 || N > kMaxRows || d <= 0 || d > kMaxWidth) return MRL_ERR_SHAPE;
  if (!is_float_type(x_dtype) || !is_float_type(weight_dtype) || !(is_float_type(y_dtype) || y_dtype == MRL_E4M3)) return MRL_ERR_DTYPE;
  if (residual != nullptr && !(residual_dtype == x_dtype || residual_dtype == MRL_F32)) return MRL_ERR_DTYPE;
  if (!(eps > 0.f && eps < 1e30f) || (scale_block != 0 && (scale_block != 128 || y_dtype != MRL_E4M3))) return MRL_ERR_CONFIG;
  if (N == 0) return MRL_OK;
  if (!x || !weight || !out_y || (residual != nullptr) != (out_sum != nullptr) || (y_dtype == MRL_E4M3) != (out_scale != nullptr))
    return MRL_ERR_NULL;
  const int rc = require_gfx950();
  if (rc != MRL_OK) return rc;
  const NormArgs a = {x, residual, weight, token_mask, N, d, eps, weight_dtype == MRL_BF16, y_dtype, scale_block, out_sum, out_y, out_scale};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (x_dtype == MRL_BF16) {
    if (residual == nullptr) go_norm<true, 0>(a, s);
    else if (residual_dtype == MRL_BF16) go_norm<true, 1>(a, s);
    else go_norm<true, 2>(a, s);
  } else if (residual == nullptr) {
    go_norm<false, 0>(a, s);
  } else {
    go_norm<false, 2>(a, s);
  }
  return hipGetLastError() == hipSuccess ? MRL_OK : MRL_ERR_DEVICE;
}

extern "C" size_t mrl_rms_norm_backward_workspace(int64_t N, int32_t d) {
  if (N < 0 || N > kMaxRows || d <= 0 || d > kMaxWidth) return 0;
  return (size_t)round_up((int64_t)back_blocks(N, d) * round_up(d, 4) * 4, 256);
}

extern "C" int mrl_rms_norm_backward(const void* dy, const void* h, const void* weight, const void* d_residual, const uint8_t* token_mask,
                                     int64_t N, int32_t d, float eps, int32_t dy_dtype, int32_t h_dtype, int32_t weight_dtype, int32_t dx_dtype,
                                     int32_t accumulate_dw, void* out_dx, float* out_dweight, void* workspace, size_t workspace_bytes, void* stream) {
  if (N < 0 || N > kMaxRows || d <= 0 || d > kMaxWidth) return MRL_ERR_SHAPE;
  if (!is_float_type(dy_dtype) || !is_float_type(h_dtype) || !is_float_type(weight_dtype) || !is_float_type(dx_dtype)) return MRL_ERR_DTYPE;
  if (!(eps > 0.f && eps < 1e30f) || (accumulate_dw != 0 && accumulate_dw != 1)) return MRL_ERR_CONFIG;
  if ((N > 0 && (!dy || !h || !weight || !out_dx)) || (N == 0 && !out_dweight && !out_dx)) return MRL_ERR_NULL;
  if (out_dweight != nullptr && N > 0 &&
      (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < mrl_rms_norm_backward_workspace(N, d)))
    return MRL_ERR_WORKSPACE;
  if (N == 0 && (out_dweight == nullptr || accumulate_dw)) return MRL_OK;
  const int rc = require_gfx950();
  if (rc != MRL_OK) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int ld = (int)round_up(d, 4), blocks = N > 0 ? back_blocks(N, d) : 0;
  float* parts = out_dweight != nullptr ? static_cast<float*>(workspace) : nullptr;
  if (N > 0) {
    const NormBackArgs a = {dy, h, weight, d_residual, token_mask, N, d, eps, weight_dtype == MRL_BF16, dx_dtype == MRL_BF16, out_dx, parts, ld};
    if (h_dtype == MRL_BF16) { if (dy_dtype == MRL_BF16) go_back<true, true>(a, s); else go_back<true, false>(a, s); }
    else { if (dy_dtype == MRL_BF16) go_back<false, true>(a, s); else go_back<false, false>(a, s); }
  }
  if (out_dweight != nullptr)                            // (of no rows: zeros)
    hipLaunchKernelGGL(k_rms_norm_dw, dim3((unsigned)((d + 15) / 16)), dim3(256), 0, s, parts, blocks, ld, d, accumulate_dw, out_dweight);
  return hipGetLastError() == hipSuccess ? MRL_OK : MRL_ERR_DEVICE;
}
