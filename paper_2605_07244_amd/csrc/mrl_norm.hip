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
  int64_t N; int d; float eps, inv_d;
  int w_bf16, y_type /*mrl_dtype*/, scale_block;
  void* sum; void* y; float* scale;
};

// Sum (or maximum) over the kT threads that share a row, a part of a wave or some waves; `sh`: a slot per wave, used by nothing else between two barriers.
template <int kT> __device__ inline float group_sum(float x, float* sh) {
  x = lanes_sum<(kT < 64 ? kT : 64)>(x);
  if (kT <= 64) return x;
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < kT / 64; ++w) s += sh[w];
  return s;
}
template <int kT> __device__ inline uint32_t group_max(uint32_t x, uint32_t* sh) {
  x = lanes_max<(kT < 64 ? kT : 64)>(x);
  if (kT <= 64) return x;
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  uint32_t m = 0;
#pragma unroll
  for (int w = 0; w < kT / 64; ++w) m = larger(m, sh[w]);
  return m;
}

// A thread's columns of one row: its i-th eight begin at column (i kT + t) 8.
template <int kT, bool kBf16> __device__ inline void load_eight(Eight<kBf16>& v, const void* row, const Columns& c, int d) {
  if (kT == 8 && d < 8) v.load_short(row, d); else v.load(row, c);       // (eight threads take rows of up to 64 columns)
}
template <int kT> __device__ inline void load_weights(const void* w, bool bf16, const Columns& c, int d, float (&out)[8]) {
  if (bf16) {
    Eight<true> v;
    load_eight<kT>(v, w, c, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = v[e];
  } else {
    Eight<false> v;
    load_eight<kT>(v, w, c, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = v[e];
  }
}

// Largest magnitude / 448, rounded as the division is: a product and a step that corrects it.
__device__ inline float scale_of(uint32_t most) {
  constexpr float kInverse = 1.f / kE4m3Max;
  const float x = __uint_as_float(most), q = x * kInverse;
  return x < INFINITY ? fmaf(fmaf(-q, kE4m3Max, x), kInverse, q) : x;
}

// kT threads take a row, each kNV times eight elements; below 64 threads a workgroup of 256 takes several.  kRes: 0 no residual, 1 bf16, 2 float.
// Memory bounds it: 65536 rows of 2048 with a residual, bf16, 178 us, 6.0 TB/s; 500000 of 128 86 us, 5.9; 32768 of 4096, a third scored, 133 us, 5.4.  Two
// vectors a thread at most, and a workgroup to a row: 5000 rows of 4096 in a wave each 34 us, in 128, 256 and 512 threads 32, 28 and 29.
// h is stored past the caches: the next layer reads y, and h is read in the backward pass (7812 rows of 4096 and a kernel that reads y: 71 us with
// both kept, 66 with h streamed, 67 with both streamed; 15625 rows 137, 136 and 139).
template <bool kXBf16, int kRes, int kT, int kNV>
__global__ __launch_bounds__(kT < 64 ? 256 : kT) void k_rms_norm(NormArgs a) {
  __shared__ float sh_sum[16];
  __shared__ uint32_t sh_max[16];
  constexpr int kRows = kT < 64 ? 256 / kT : 1;
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kRows + threadIdx.x / kT;
  if (row >= a.N) return;                               // (all of a row's threads)
  const int t = threadIdx.x % kT, d = a.d;
  const int scales = a.scale_block ? (d + 127) / 128 : 1;
  const char* x = static_cast<const char*>(a.x) + row * d * (kXBf16 ? 2 : 4);
  const char* res = static_cast<const char*>(a.residual) + row * d * (kRes == 1 ? 2 : 4);
  char* sum = static_cast<char*>(a.sum) + row * d * (kRes == 1 ? 2 : 4);
  char* y = static_cast<char*>(a.y) + row * d * (a.y_type == MRL_F32 ? 4 : a.y_type == MRL_BF16 ? 2 : 1);
  // Rows without a residual have few bytes under way for their latencies: the weights come with the row and not behind its sum, and
  // a row that is not scored leaves at once (98341 rows of 2048, us: bf16 152 -> 137, e4m3 141 -> 130, 34 % scored 146 -> 115).  With a residual
  // the registers and the burst of zeros cost more than that (34 % scored, 32768 rows of 4096 and 25906 of 7002: 135 -> 138 us, 385 -> 393).
  constexpr bool kLight = kRes == 0 && kT >= 64;
  const bool scored = a.mask == nullptr || a.mask[row] != 0;
  if (kLight && !scored) {                              // (all of a row's threads again)
    const float zero[8] = {};
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      const Columns c((i * kT + t) * 8, d);
      if (a.y_type == MRL_E4M3) store_eight_e4m3(y, c, d, zero); else store_eight(y, a.y_type == MRL_BF16, c, d, zero);
    }
    if (a.y_type == MRL_E4M3)
      for (int k = t; k < scales; k += kT) a.scale[row * scales + k] = scale_of(kScaleLeast);
    return;
  }
  float h[kNV][8], w[kNV][8];
  if (scored) {
    Eight<kXBf16> xv[kNV];
    Eight<kRes == 1> rv[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      const Columns c((i * kT + t) * 8, d);
      load_eight<kT>(xv[i], x, c, d);
      if (kRes) load_eight<kT>(rv[i], res, c, d);
    }
    if (kLight) {
#pragma unroll
      for (int i = 0; i < kNV; ++i) load_weights<kT>(a.w, a.w_bf16, Columns((i * kT + t) * 8, d), d, w[i]);
    }
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      const Columns c((i * kT + t) * 8, d);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] = e < c.skip ? 0.f : kRes ? xv[i][e] + rv[i][e] : xv[i][e];
    }
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
    if (kRes) store_eight<true>(sum, kRes == 1, Columns((i * kT + t) * 8, d), d, h[i]);
  }
  s = group_sum<kT>(s, sh_sum);
  const float r = __builtin_amdgcn_rsqf(fmaf(s, a.inv_d, a.eps));      // (the instruction is good to a step of fp32)
#pragma unroll
  for (int i = 0; i < kNV; ++i) {
    const Columns c((i * kT + t) * 8, d);
    if (!kLight) load_weights<kT>(a.w, a.w_bf16, c, d, w[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[i][e] = scored && e >= c.skip ? h[i][e] * r * w[i][e] : 0.f;
  }
  if (a.y_type != MRL_E4M3) {
#pragma unroll
    for (int i = 0; i < kNV; ++i) store_eight(y, a.y_type == MRL_BF16, Columns((i * kT + t) * 8, d), d, h[i]);
    return;
  }
  uint32_t most[kNV];
#pragma unroll
  for (int i = 0; i < kNV; ++i) {
    most[i] = kScaleLeast;
#pragma unroll
    for (int e = 0; e < 8; ++e) most[i] = larger(most[i], magnitude(h[i][e]));
  }
  if (kT > 8 && a.scale_block) {                        // 128 columns are 16 lanes (and a row of up to 64 is one block)
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      most[i] = lanes_max<16>(most[i]);
      const int block = (i * kT + t) / 16;
      if ((t & 15) == 0 && block < scales) a.scale[row * scales + block] = scale_of(most[i]);
    }
  } else {
#pragma unroll
    for (int i = 1; i < kNV; ++i) most[0] = larger(most[0], most[i]);
    most[0] = group_max<kT>(most[0], sh_max);
#pragma unroll
    for (int i = 1; i < kNV; ++i) most[i] = most[0];
    if (t == 0) a.scale[row] = scale_of(most[0]);
  }
#pragma unroll
  for (int i = 0; i < kNV; ++i) {
    // y / scale: a product with the reciprocal and a step that corrects it, as exact as a division and a third of its instructions (the product alone is
    // off by another half a step of fp32, and twice as many codes fall on the other side of a rounding as need be).  Infinite scales: reciprocal and
    // divisor zero leave finite values at zero.
    const float scale = scale_of(most[i]), inverse = __builtin_amdgcn_rcpf(scale), divisor = scale < INFINITY ? scale : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float q = h[i][e] * inverse;
      h[i][e] = fmaf(fmaf(-q, divisor, h[i][e]), inverse, q);
    }
    store_eight_e4m3(y, Columns((i * kT + t) * 8, d), d, h[i]);
  }
}

struct NormBackArgs {
  const void* dy; const void* h; const void* w; const void* d_residual; const uint8_t* mask;
  int64_t N; int d; float eps, inv_d;
  int w_bf16, dx_bf16;
  void* dx; float* parts /*[gridDim.x][ld] | nullptr*/; int ld;
};

// What a thread holds of a row.
template <bool kHBf16, bool kDyBf16, int kT, int kNV> struct BackRow {
  Eight<kHBf16> h[kNV], res[kNV];
  Eight<kDyBf16> dy[kNV];
  bool scored;
  __device__ void load(const NormBackArgs& a, int64_t row, bool is_scored, int t) {
    scored = is_scored;
    const int64_t at = row * a.d;
    const char* h_row = static_cast<const char*>(a.h) + at * (kHBf16 ? 2 : 4);
    const char* dy_row = static_cast<const char*>(a.dy) + at * (kDyBf16 ? 2 : 4);
    const char* res_row = static_cast<const char*>(a.d_residual) + at * (kHBf16 ? 2 : 4);
    if (is_scored) {
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        const Columns c((i * kT + t) * 8, a.d);
        load_eight<kT>(h[i], h_row, c, a.d);
        load_eight<kT>(dy[i], dy_row, c, a.d);
      }
    }
    if (a.d_residual != nullptr) {
#pragma unroll
      for (int i = 0; i < kNV; ++i) load_eight<kT>(res[i], res_row, Columns((i * kT + t) * 8, a.d), a.d);
    }
  }
};

// The rows of a workgroup one after the other (up to 64 threads a row: several side by side), the next one's elements on their way while one is
// worked on, and the mask of the one behind it; the columns' sums of dy u stay in registers until the last row.  Then the rows that were
// side by side are added in LDS, in their order, and the workgroup writes one row of partial sums.
// Memory bounds it in long calls (80000 rows of 2048 with d_residual 229 us, 5.7 TB/s; 500000 of 128 104 us, 4.9), in short ones the latency of a workgroup's rows
// (400 of 1536 in 5.1 us; 3001 of 713 in 12.4, of which the waves' sums in LDS are a part: they go in one after the other, a column at a time, and a lane waits for each).
// In round k the workgroups take consecutive rows, turned by k times a golden section of their number: sequences of as many slots as there are
// workgroups, whose heads are scored and whose tails are not, would else give some of them scored rows only.
template <bool kHBf16, bool kDyBf16, int kT, int kNV>
__global__ __launch_bounds__(kT <= 64 ? 256 : kT) void k_rms_norm_back(NormBackArgs a) {
  extern __shared__ float lds[];                        // kT <= 64: [d] sums; else two sets of two sums a wave
  constexpr int kRows = kT <= 64 ? 256 / kT : 1;
  const int t = threadIdx.x % kT, side = threadIdx.x / kT, d = a.d;
  const int slots = (int)gridDim.x * kRows, slot = (int)blockIdx.x * kRows + side;
  const int turn_by = (int)(slots * 0.618f), rounds = (int)((a.N + slots - 1) / slots);
  float acc[kNV][8], w[kNV][8];                         // (weights stay in registers, too: every row needs them twice)
#pragma unroll
  for (int i = 0; i < kNV; ++i) {
    load_weights<kT>(a.w, a.w_bf16, Columns((i * kT + t) * 8, d), d, w[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[i][e] = 0.f;
  }
  int64_t base = 0;
  int place = slot;
  auto next_row = [&]() -> int64_t {                    // of the next round, or -1
    const int64_t row = base + place;
    base += slots;
    place += turn_by;
    if (place >= slots) place -= slots;
    return row < a.N ? row : -1;
  };
  auto mask_of = [&](int64_t row) -> int { return row < 0 ? 0 : a.mask == nullptr ? 1 : a.mask[row]; };
  constexpr bool kAhead = kNV < 4;                      // (two rows of more do not fit the registers)
  BackRow<kHBf16, kDyBf16, kT, kNV> now, next;
  int64_t row = next_row(), row1 = next_row();
  int mask0 = mask_of(row), mask1 = mask_of(row1), turn = 0;
  auto is_scored = [](int m) { return (kT < 64 ? m : __builtin_amdgcn_readfirstlane(m)) != 0; };     // (one row a wave: a scalar condition)
  if (kAhead && row >= 0) now.load(a, row, is_scored(mask0), t);
  for (int k = 0; k < rounds; ++k) {
    const int64_t row2 = next_row();
    const int mask2 = mask_of(row2);
    if (kAhead && row1 >= 0) next.load(a, row1, is_scored(mask1), t);
    if (!kAhead && row >= 0) now.load(a, row, is_scored(mask0), t);
    if (row >= 0) {                                     // (with more waves than one a row, the workgroup is of one mind)
      char* dx = static_cast<char*>(a.dx) + row * d * (a.dx_bf16 ? 2 : 4);
      float r = 0.f, along = 0.f;
      if (now.scored) {
        float hh = 0.f, gh = 0.f;
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
          const Columns c((i * kT + t) * 8, d);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (e < c.skip) continue;                   // (a column of another thread)
            hh = fmaf(now.h[i][e], now.h[i][e], hh);
            gh = fmaf(now.dy[i][e] * w[i][e], now.h[i][e], gh);
          }
        }
        hh = lanes_sum<(kT < 64 ? kT : 64)>(hh);
        gh = lanes_sum<(kT < 64 ? kT : 64)>(gh);
        if (kT > 64) {                                  // (two sets of slots in turn from one scored row to the next: one barrier each)
          float* sh = lds + turn * 32;
          turn ^= 1;
          if ((threadIdx.x & 63) == 0) { sh[threadIdx.x >> 6] = hh; sh[16 + (threadIdx.x >> 6)] = gh; }
          __syncthreads();
          hh = gh = 0.f;
#pragma unroll
          for (int v = 0; v < kT / 64; ++v) { hh += sh[v]; gh += sh[16 + v]; }
        }
        r = __builtin_amdgcn_rsqf(fmaf(hh, a.inv_d, a.eps));
        along = gh * r * a.inv_d;
      }
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        float out[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          out[e] = 0.f;
          if (now.scored) {
            const float u = now.h[i][e] * r;
            acc[i][e] = fmaf(now.dy[i][e], u, acc[i][e]);
            out[e] = r * (now.dy[i][e] * w[i][e] - u * along);
          }
          if (a.d_residual != nullptr) out[e] += now.res[i][e];
        }
        store_eight(dx, a.dx_bf16, Columns((i * kT + t) * 8, d), d, out);
      }
    }
    if (kAhead) now = next;
    row = row1; row1 = row2; mask0 = mask1; mask1 = mask2;
  }
  if (a.parts == nullptr) return;
  float* part = a.parts + (int64_t)blockIdx.x * a.ld;
  if (kT > 64) {
#pragma unroll
    for (int i = 0; i < kNV; ++i) store_eight(part, false, Columns((i * kT + t) * 8, d), d, acc[i]);
    return;
  }
#pragma unroll
  for (int i = 0; i < kNV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
      for (int off = kT; off < 64; off <<= 1) acc[i][e] += __shfl_xor(acc[i][e], off);
    }
  const int wave = threadIdx.x >> 6;
  for (int v = 0; v < 4; ++v) {
    if (wave == v && (threadIdx.x & 63) < kT) {
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        const Columns c((i * kT + t) * 8, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (!c.own(e, d)) continue;
          const float sum = v > 0 ? lds[c.at + e] + acc[i][e] : acc[i][e];
          if (v < 3) lds[c.at + e] = sum; else part[c.at + e] = sum;
        }
      }
    }
    __syncthreads();
  }
}

// dw[c] = (or +=) sum of the workgroups' partial sums, in fp64 in a fixed order: kDwLanes times four columns a workgroup, the other threads along
// the partials.  Latency bounds it: 512 partials of 2048 columns 4.8 us.  (One, two and four lanes: the whole backward pass of 400 rows of 1536 9.7, 8.4 and 8.2 us.)
constexpr int kDwLanes = 4;
__global__ __launch_bounds__(256) void k_rms_norm_dw(const float* parts, int n_parts, int ld, int d, int accumulate, float* dw) {
  __shared__ double sh[4][4 * kDwLanes];
  const int at = threadIdx.x % kDwLanes, c0 = (blockIdx.x * kDwLanes + at) * 4, lane = threadIdx.x & 63;
  constexpr int kAlong = 256 / kDwLanes;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  if (c0 < ld) {
    for (int p0 = threadIdx.x / kDwLanes; p0 < n_parts; p0 += kAlong * 4) {
      float4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        v[k] = p0 + kAlong * k < n_parts ? *reinterpret_cast<const float4*>(parts + (int64_t)(p0 + kAlong * k) * ld + c0) : float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 4; ++k) { s[0] += (double)v[k].x; s[1] += (double)v[k].y; s[2] += (double)v[k].z; s[3] += (double)v[k].w; }
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int off = kDwLanes; off < 64; off <<= 1) s[k] += __shfl_xor(s[k], off);
    if (lane < kDwLanes) sh[threadIdx.x >> 6][lane * 4 + k] = s[k];
  }
  __syncthreads();
  const int c = blockIdx.x * 4 * kDwLanes + threadIdx.x;
  if (threadIdx.x < 4 * kDwLanes && c < d) {
    double total = (sh[0][threadIdx.x] + sh[1][threadIdx.x]) + (sh[2][threadIdx.x] + sh[3][threadIdx.x]);
    if (accumulate) total += (double)dw[c];
    dw[c] = (float)total;
  }
}

constexpr int kMaxWidth = 16384;                         // 1024 threads, 16 elements each

// Threads that share a row, and how many times eight elements each takes.
struct Shape { int threads, vectors; };
Shape norm_shape(int d) {
  const int v = (d + 7) / 8;
  if (v <= 64) return {v <= 8 ? 8 : v <= 16 ? 16 : v <= 32 ? 32 : 64, 1};
  if (v <= 128) return {64, 2};
  if (v <= 256) return {v <= 192 ? 192 : 256, 1};
  if (v <= 512) return {256, 2};
  if (v <= 1024) return {512, 2};
  return {1024, 2};
}
// Up to 128 vectors of eight a wave or a part of one takes a row, several of them side by side; above, as many waves as the row has vectors for, with one each: idle
// lanes cost more than barriers (65104 rows of 1536 in 256 and in 192 threads 182 and 153 us, 27901 of 3584 in 256 threads with two vectors and in 448
// with one 173 and 150).
Shape back_shape(int d) {
  const int v = (d + 7) / 8;
  if (v <= 128) return {v <= 8 ? 8 : v <= 16 ? 16 : v <= 32 ? 32 : 64, v <= 64 ? 1 : 2};
  if (v <= 512) return {v <= 192 ? 192 : (v + 63) / 64 * 64, 1};
  return {512, v <= 1024 ? 2 : 4};
}
int rows_side_by_side(const Shape& s) { return s.threads <= 64 ? 256 / s.threads : 1; }
// Rows above 8192 columns, a workgroup's one row under way at a time: 134 M elements as rows of 4096, 8192, 12288 and 16384 in bf16 162, 164, 201 and 182 us (at 5.9 TB/s 137), with
// d_residual 200, 199, 230 and 221 (182); float 307, 302, 304 and 317 (273).  Calls of few such rows wait for them: 300 of 16384 22 us, 2000 50 (33).
// Workgroups: two or more rows each, and as many as cover the latencies of a row without more rows under way than the memory takes well: 80000 rows of 2048,
// us, with 256, 512, 768, 1024 and 1280 workgroups: 351, 229, 238, 259, 282.  The partial sums of many are worth it to long calls only: rows of 4096 in
// 512 threads, with 256 and 512 workgroups: 1000 rows 13.8 and 16.2, 4000 28.8 and 31.6, 24414 156 and 154; of 1536 in 192 threads, with 512 and 1024: 4000 rows
// 17.3 and (768) 18.2, 65104 171 and 157.
// A long call without d_residual, which has fewer bytes under way for each of them, takes twice as many below 512 threads: 78125 rows of 2048 211 and 185 us, 62500 of 2560
// 207 and 187, 468750 of 128 111 and 81; with d_residual 229 and 258, 235 and 260; 39062 rows of 4096 184 and 198 without.  Rows that share a wave take three a compute
// unit with it (468750 of 128 with 512, 768 and 1024: 120, 101, 104).
int back_blocks(int64_t N, int d, bool has_residual) {
  const Shape sh = back_shape(d);
  const int64_t b = (N + 2 * rows_side_by_side(sh) - 1) / (2 * rows_side_by_side(sh));
  const bool is_long = N >= 16384;
  int most = 512;
  if (sh.threads == 512 && sh.vectors > 1) most = 256;
  else if (!is_long) most = sh.threads >= 384 ? 256 : 512;
  else if (sh.threads == 192 || (sh.threads < 512 && sh.vectors == 1 && !has_residual)) most = 1024;
  else if (sh.threads < 64) most = 768;
  return (int)(b < most ? b : most);
}

constexpr int64_t kMostWide = 1 << 21;                   // workgroups along x: a launch has fewer than 2^32 threads there

template <bool kXBf16, int kRes, int kT, int kNV> void go_norm_shape(const NormArgs& a, hipStream_t s) {
  constexpr int kRows = kT < 64 ? 256 / kT : 1;
  const int64_t groups = (a.N + kRows - 1) / kRows, wide = groups < kMostWide ? groups : kMostWide;
  hipLaunchKernelGGL((k_rms_norm<kXBf16, kRes, kT, kNV>), dim3((unsigned)wide, (unsigned)((groups + wide - 1) / wide)), dim3(kT < 64 ? 256 : kT), 0, s, a);
}
template <bool kXBf16, int kRes> void go_norm(const NormArgs& a, hipStream_t s) {
  const Shape sh = norm_shape(a.d);
  switch (sh.threads * 8 + sh.vectors) {
    case 8 * 8 + 1: go_norm_shape<kXBf16, kRes, 8, 1>(a, s); break;
    case 16 * 8 + 1: go_norm_shape<kXBf16, kRes, 16, 1>(a, s); break;
    case 32 * 8 + 1: go_norm_shape<kXBf16, kRes, 32, 1>(a, s); break;
    case 64 * 8 + 1: go_norm_shape<kXBf16, kRes, 64, 1>(a, s); break;
    case 64 * 8 + 2: go_norm_shape<kXBf16, kRes, 64, 2>(a, s); break;
    case 192 * 8 + 1: go_norm_shape<kXBf16, kRes, 192, 1>(a, s); break;
    case 256 * 8 + 1: go_norm_shape<kXBf16, kRes, 256, 1>(a, s); break;
    case 256 * 8 + 2: go_norm_shape<kXBf16, kRes, 256, 2>(a, s); break;
    case 512 * 8 + 2: go_norm_shape<kXBf16, kRes, 512, 2>(a, s); break;
    default: go_norm_shape<kXBf16, kRes, 1024, 2>(a, s); break;
  }
}

template <bool kHBf16, bool kDyBf16> void go_back(const NormBackArgs& a, hipStream_t s) {
  const Shape sh = back_shape(a.d);
  const bool waves = sh.threads <= 64;
  const dim3 grid((unsigned)back_blocks(a.N, a.d, a.d_residual != nullptr)), block(waves ? 256 : sh.threads);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, waves ? (size_t)a.d * 4 : 64 * 4, s, a); };
  switch (sh.threads * 8 + sh.vectors) {
    case 8 * 8 + 1: go(k_rms_norm_back<kHBf16, kDyBf16, 8, 1>); break;
    case 16 * 8 + 1: go(k_rms_norm_back<kHBf16, kDyBf16, 16, 1>); break;
    case 32 * 8 + 1: go(k_rms_norm_back<kHBf16, kDyBf16, 32, 1>); break;
    case 64 * 8 + 1: go(k_rms_norm_back<kHBf16, kDyBf16, 64, 1>); break;
    case 64 * 8 + 2: go(k_rms_norm_back<kHBf16, kDyBf16, 64, 2>); break;
    case 192 * 8 + 1: go(k_rms_norm_back<kHBf16, kDyBf16, 192, 1>); break;
    case 256 * 8 + 1: go(k_rms_norm_back<kHBf16, kDyBf16, 256, 1>); break;
    case 320 * 8 + 1: go(k_rms_norm_back<kHBf16, kDyBf16, 320, 1>); break;
    case 384 * 8 + 1: go(k_rms_norm_back<kHBf16, kDyBf16, 384, 1>); break;
    case 448 * 8 + 1: go(k_rms_norm_back<kHBf16, kDyBf16, 448, 1>); break;
    case 512 * 8 + 1: go(k_rms_norm_back<kHBf16, kDyBf16, 512, 1>); break;
    case 512 * 8 + 2: go(k_rms_norm_back<kHBf16, kDyBf16, 512, 2>); break;
    default: go(k_rms_norm_back<kHBf16, kDyBf16, 512, 4>); break;
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
  if (!(eps >= 1e-30f && eps < 1e30f) || (scale_block != 0 && (scale_block != 128 || y_dtype != MRL_E4M3))) return MRL_ERR_CONFIG;
  if (N == 0) return MRL_OK;
  if (!x || !weight || !out_y || (residual != nullptr) != (out_sum != nullptr) || (y_dtype == MRL_E4M3) != (out_scale != nullptr))
    return MRL_ERR_NULL;
  const int rc = require_gfx950();
  if (rc != MRL_OK) return rc;
  const NormArgs a = {x, residual, weight, token_mask, N, d, eps, 1.f / (float)d, weight_dtype == MRL_BF16, y_dtype, scale_block, out_sum, out_y, out_scale};
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
  return (size_t)round_up((int64_t)back_blocks(N, d, false) * round_up(d, 4) * 4, 256);     // (no fewer than with d_residual)
}

extern "C" int mrl_rms_norm_backward(const void* dy, const void* h, const void* weight, const void* d_residual, const uint8_t* token_mask,
                                     int64_t N, int32_t d, float eps, int32_t dy_dtype, int32_t h_dtype, int32_t weight_dtype, int32_t dx_dtype,
                                     int32_t accumulate_dw, void* out_dx, float* out_dweight, void* workspace, size_t workspace_bytes, void* stream) {
  if (N < 0 || N > kMaxRows || d <= 0 || d > kMaxWidth) return MRL_ERR_SHAPE;
  if (!is_float_type(dy_dtype) || !is_float_type(h_dtype) || !is_float_type(weight_dtype) || !is_float_type(dx_dtype)) return MRL_ERR_DTYPE;
  if (!(eps >= 1e-30f && eps < 1e30f) || (accumulate_dw != 0 && accumulate_dw != 1)) return MRL_ERR_CONFIG;
  if (N > 0 && (!dy || !h || !weight || !out_dx)) return MRL_ERR_NULL;
  if (out_dweight != nullptr && N > 0 &&
      (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < mrl_rms_norm_backward_workspace(N, d)))
    return MRL_ERR_WORKSPACE;
  if (N == 0 && (out_dweight == nullptr || accumulate_dw)) return MRL_OK;
  const int rc = require_gfx950();
  if (rc != MRL_OK) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int ld = (int)round_up(d, 4), blocks = N > 0 ? back_blocks(N, d, d_residual != nullptr) : 0;
  float* parts = out_dweight != nullptr ? static_cast<float*>(workspace) : nullptr;
  if (N > 0) {
    const NormBackArgs a = {dy, h, weight, d_residual, token_mask, N, d, eps, 1.f / (float)d, weight_dtype == MRL_BF16, dx_dtype == MRL_BF16, out_dx, parts, ld};
    if (h_dtype == MRL_BF16) { if (dy_dtype == MRL_BF16) go_back<true, true>(a, s); else go_back<true, false>(a, s); }
    else { if (dy_dtype == MRL_BF16) go_back<false, true>(a, s); else go_back<false, false>(a, s); }
  }
  if (out_dweight != nullptr)                            // (of no rows: zeros)
    hipLaunchKernelGGL(k_rms_norm_dw, dim3((unsigned)((d + 4 * kDwLanes - 1) / (4 * kDwLanes))), dim3(256), 0, s, parts, blocks, ld, d, accumulate_dw, out_dweight);
  return hipGetLastError() == hipSuccess ? MRL_OK : MRL_ERR_DEVICE;
}
