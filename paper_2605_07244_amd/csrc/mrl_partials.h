// The forward kernel's partial sums, added per row by the row epilogues of the two losses.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mrl {

__device__ inline int valid_rows(const int64_t* n_scored, int64_t chunk_start, int chunk_rows) {
  const int64_t r = *n_scored - chunk_start;
  return r < 0 ? 0 : (r > chunk_rows ? chunk_rows : (int)r);
}

// Block = 64 rows x 64 partial lanes: see merge_partials.
constexpr int EPI_ROWS = 64;
constexpr int EPI_THREADS = 1024;
constexpr int EPI_LANES = EPI_THREADS / (EPI_ROWS / 4);
// K loads of a thread's partials, in flight together: every EPI_LANES-th from q on, of which `left` (of the block's numbering) remain.
template <int K, bool ALL> __device__ __forceinline__ void add_partials(const float* q, int64_t step, int left, float4& s) {
  float4 v[K];
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = *reinterpret_cast<const float4*>(ALL || k * EPI_LANES < left ? q + k * step : q);
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (ALL || k * EPI_LANES < left) { s.x += v[k].x; s.y += v[k].y; s.z += v[k].z; s.w += v[k].w; }
}
// Sum over all partials of this block's 64 rows; the result is valid in threads 0 .. 63 (one row
// each).  Fixed order.  src points at the block's first row; rows beyond the valid ones hold
// whatever the buffer held.  All threads must call it.
__device__ inline float merge_partials(const float* src, int64_t stride, int n_partials, float4 (&sh)[EPI_LANES][EPI_ROWS / 4]) {
  const int quad = threadIdx.x & 15, part = threadIdx.x >> 4;
  const int64_t step = stride * EPI_LANES;
  const float* q = src + (part < n_partials ? part : 0) * stride + quad * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  int rest = n_partials;                              // from the block's first on
  for (; rest >= EPI_LANES * 8; rest -= EPI_LANES * 8, q += 8 * step) add_partials<8, true>(q, step, 0, s);
  const int left = rest - part;                       // the thread's first is `part` of them
  if (rest > EPI_LANES * 4) add_partials<8, false>(q, step, left, s);
  else if (rest > EPI_LANES * 2) add_partials<4, false>(q, step, left, s);
  else if (rest > EPI_LANES) add_partials<2, false>(q, step, left, s);
  else if (left > 0) add_partials<1, true>(q, step, 0, s);
  __syncthreads();                                  // an earlier merge has been read
  sh[part][quad] = s;
  __syncthreads();
  // 16 waves, one row per lane, 4 lanes' sums each; then the 16 wave sums by the first wave
  const int row = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto cell = [&](int l) -> float& { return reinterpret_cast<float*>(&sh[l][0])[row]; };
  const float t = (cell(4 * wave) + cell(4 * wave + 1)) + (cell(4 * wave + 2) + cell(4 * wave + 3));
  __syncthreads();
  cell(wave) = t;
  __syncthreads();
  float sum = 0.f;
  if (wave == 0) {
#pragma unroll
    for (int w = 0; w < EPI_THREADS / 64; ++w) sum += cell(w);
  }
  return sum;
}

}  // namespace mrl
