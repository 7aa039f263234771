// Distillation from a teacher's top log-probs: what surrounds the products of the loss.  Row n has alternatives j = 1 .. k with ids v_j and log-probs t_j,
// q_j = exp t_j (renormalised: over their sum), m = sum q_j, p = softmax(z / T):
//   kl = sum_j q_j (log q_j - log p[v_j])          L = T^2 sum_n w_n kl_n          dz = w T (m p - q)
// With the forward launch's stash e = 2^(z log2(e) / T - c) and its sum S, p = e / S and
//   dz = (w T m / S) (e - S (q / m)):  the stored row, changed at k places, times a scalar per row.
// The offset c comes from the largest of the row's k logits, which are products of the row with k rows of the head, taken
// before the forward launch in fp32: the divergence needs them to more bits than the stash has.  The weights and divergences of a row are taken in
// 64 bits: a few dozen operations beside 6 d V.  What is rounded to 16 bits, and how far that takes the gradients: e (or e - S (q / m)) in the stash and the row of
// hidden states times its scale, half a step of 2^-9 each on average a third of it; dH 1.7e-3 of its norm and dW 2.4e-3, with the rounding of a bf16 output 2.4e-3 and 2.9e-3.
#include "mrl_internal.h"
#include "mrl_vec.h"

namespace mrl {
namespace {

constexpr double LN2 = 0.6931471805599453;
constexpr double kLeastMass = 1e-30;                   // of a row that counts: w T m stays a normal float for weights down to 1e-8
constexpr double kLeastScale = 0x1p-100;               // of a row: its products with ordinary hidden states stay normal floats and bf16

__device__ inline double wave_sum(double x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
  return x;
}
__device__ inline float wave_max(float x) {            // NaN is passed over
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
  return x;
}

// A slot's alternatives, by one wave, kEach to a lane: j = 64 i + lane.
template <int kEach> struct Alternatives {
  int id[kEach];                                       // -1: none
  float t[kEach];
  double q[kEach], log_q[kEach], m;
  bool any;                                            // the slot counts
  int too_large;                                       // ids that name no token though they are not negative
  __device__ void load(const DistillArgs& a, int64_t slot) {
    const int lane = threadIdx.x & 63;
    const int32_t* ids = a.ids + slot * a.k;
    const float* logp = a.logp + slot * a.k;
    too_large = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int j = 64 * i + lane;
      const bool in = j < a.k;
      const int v = ids[in ? j : 0];
      const float p = logp[in ? j : 0];                // (both under way at once)
      id[i] = in && v >= 0 && v < a.V ? v : -1;
      t[i] = id[i] >= 0 ? p : -INFINITY;
      too_large += __popcll(__ballot(in && v >= a.V));
    }
  }
  // (best: the largest t; with nothing above -infinity and no NaN, nothing counts)
  __device__ void weigh(const DistillArgs& a, float best) {
    const double shift = a.renormalize ? (double)best : 0.0;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      log_q[i] = (double)t[i] - shift;
      q[i] = id[i] >= 0 ? t[i] == -INFINITY ? 0.0 : exp(log_q[i]) : 0.0;
      sum += q[i];
    }
    m = wave_sum(sum);
    any = m != m || m >= kLeastMass;
    if (!a.renormalize) {
      // an infinite mass is no distribution's: NaN, as the quotients of infinities below
      const double nan = __builtin_nan("");
      if (m == (double)INFINITY) {
        m = nan;
#pragma unroll
        for (int i = 0; i < kEach; ++i) q[i] = id[i] >= 0 ? nan : 0.0;
      }
      return;
    }
    const double log_m = log(m), inv = 1.0 / m;
#pragma unroll
    for (int i = 0; i < kEach; ++i) { q[i] *= inv; log_q[i] -= log_m; }
    m = m != m ? m : 1.0;
  }
  __device__ float best_t() const {
    float b = t[0];
#pragma unroll
    for (int i = 1; i < kEach; ++i) b = fmaxf(b, t[i]);
    return wave_max(b);
  }
  // Per alternative its id's share of the mass, however often that is listed, and whether this is the id's first place.
  __device__ void by_id(int k, float (&share)[kEach], bool (&first)[kEach]) const {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < kEach; ++i) { share[i] = 0.f; first[i] = id[i] >= 0; }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int n = k - 64 * e < 64 ? k - 64 * e : 64;
      const float mine = (float)(q[e] / m);
      for (int l = 0; l < n; ++l) {
        const int other = __builtin_amdgcn_readlane(id[e], l);
        const float p = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), l));
#pragma unroll
        for (int i = 0; i < kEach; ++i)
          if (id[i] == other && 64 * i < k) {
            share[i] += p;
            if (64 * e + l < 64 * i + lane) first[i] = false;
          }
      }
    }
  }
};

__device__ inline float weight_of(const DistillArgs& a, int64_t slot) {
  return a.weight != nullptr ? a.weight[slot] : (float)(1.0 / (double)*a.n_scored);
}

// A wave per slot: the id of its best alternative, or -1.
template <int kEach> __global__ __launch_bounds__(256) void k_distill_targets(DistillArgs a) {
  const int64_t n = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (n >= a.N) return;
  int target = -1;
  if (a.mask == nullptr || a.mask[n] != 0) {
    Alternatives<kEach> alt;
    alt.load(a, n);
    const float best = alt.best_t();
    alt.weigh(a, best);
    // the lowest lane that has it (of NaN alone, where the largest is NaN if every lane holds one and else -infinity: any alternative)
#pragma unroll
    for (int i = kEach - 1; i >= 0; --i) {
      const unsigned long long has = __ballot(alt.id[i] >= 0 && (alt.t[i] == best || !(best > -INFINITY)));
      if (has != 0) target = __builtin_amdgcn_readlane(alt.id[i], __builtin_ctzll(has));
    }
    if (!alt.any) target = -1;
  }
  if ((threadIdx.x & 63) == 0) a.targets[n] = target;
}

// ----------------------------------------------------------------------------
// bf16: the alternatives' logits.  A workgroup per row, its waves taking eight alternatives at a time, a lane eight columns, sums in fp32.  Bound by the rows of the
// head that it reads, k of them per token with little in common: 8192 rows, k = 64, d = 4096 584 us, 4.3 GB at 7.4 TB/s (3 % of the call).  The logits that
// the forward launch makes would need no such reads, but it meets a row's alternatives in as many tiles.
// ----------------------------------------------------------------------------
constexpr int kTogether = 8;
__global__ __launch_bounds__(256) void k_distill_logits(DistillArgs a) {
  __shared__ float most[4];
  const int64_t r = blockIdx.x;
  if (r >= valid_rows(a.n_scored, a.chunk_start, a.chunk_rows)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t slot = a.row_index[a.chunk_start + r];
  const u32x4* const h = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.H) + slot * a.d);
  const int32_t* const ids = a.ids + slot * a.k;
  const float* const logp = a.logp + slot * a.k;
  const int vectors = a.d / 8;
  float largest = -INFINITY;
  for (int j0 = wave * kTogether; j0 < a.k; j0 += 4 * kTogether) {
    const u32x4* w[kTogether];
    bool there[kTogether];
#pragma unroll
    for (int i = 0; i < kTogether; ++i) {
      const int id = j0 + i < a.k ? ids[j0 + i] : -1;
      there[i] = id >= 0 && id < a.V;
      w[i] = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.W) + (int64_t)(there[i] ? id : 0) * a.d);
    }
    float acc[kTogether] = {};
    for (int c = lane; c < vectors; c += 64) {
      const u32x4 u = h[c];
      u32x4 b[kTogether];
#pragma unroll
      for (int i = 0; i < kTogether; ++i) b[i] = w[i][c];
#pragma unroll
      for (int i = 0; i < kTogether; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[i] = fmaf(bf16_low(u[e]), bf16_low(b[i][e]), acc[i]);
          acc[i] = fmaf(bf16_high(u[e]), bf16_high(b[i][e]), acc[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < kTogether; ++i) {
      const float z = lanes_sum<64>(acc[i]);
      if (j0 + i >= a.k) continue;
      if (lane == 0) a.zk[r * a.k + j0 + i] = z;
      if (there[i] && logp[j0 + i] != -INFINITY) largest = fmaxf(largest, z);
    }
  }
  if (lane == 0) most[wave] = largest;
  __syncthreads();
  if (threadIdx.x == 0) a.zt[a.chunk_start + r] = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
}

// Behind the forward launch: what its clamp hides.  Exponentials are clamped at 2^kStashClamp2, and so are those of NaN and +infinity, which would pass for logits far
// above the alternatives'.  A workgroup per partial sum, those of kPartialRows rows of the head: where a token's reaches the clamp and the rows hold anything that is not finite, that
// token's sum is NaN.  The head is read at clamped sums only, once at most.  (Finite logits that reach the clamp beside such an entry: their row is saturated, and NaN with it.)
// (It takes 5 us of 200 rows and of 900, 19 of 8192, V = 151936: 39 MB.  A call of 200 rows, d = 1536 425 us without it and 429 with; of 900, V = 50257, d = 712 325 and 330.)
constexpr int kPartialRows = 128;
__global__ __launch_bounds__(256) void k_distill_hidden_nan(DistillArgs a) {
  const int nvalid = valid_rows(a.n_scored, a.chunk_start, a.chunk_rows);
  const int64_t v0 = (int64_t)blockIdx.x * kPartialRows;
  const int rows = a.V - v0 < kPartialRows ? (int)(a.V - v0) : kPartialRows;
  float* const sums = a.part_sum + (int64_t)blockIdx.x * a.chunk_rows;
  constexpr float clamped = 0x1p99f;                   // (half of it, however it is rounded)
  static_assert(kStashClamp2 == 100.f, "the clamp");
  bool any = false;
  for (int n = threadIdx.x; n < nvalid; n += 256) any |= sums[n] >= clamped;
  if (!__syncthreads_or(any)) return;
  const uint16_t* const w = static_cast<const uint16_t*>(a.W) + v0 * a.d;
  bool bad = false;
  for (int64_t i = threadIdx.x * 8; i < (int64_t)rows * a.d; i += 256 * 8) {
    const u32x4 x = load_any<2, u32x4>(w + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) bad |= (x[e] & 0x7f80u) == 0x7f80u || (x[e] & 0x7f800000u) == 0x7f800000u;
  }
  if (!__syncthreads_or(bad)) return;
  for (int n = threadIdx.x; n < nvalid; n += 256)
    if (sums[n] >= clamped) sums[n] = __builtin_nanf("");
}

// Behind that: a workgroup adds the partial sums of 16 rows, then a wave takes each.  (Blocks of 64 rows, four to a wave, left most of the chip idle:
// V = 151936, 200 rows, k = 32 50 us, now 14; 8192 rows, k = 64 77, now 33, 39 MB of partial sums and the alternatives' logits.)
constexpr int kRows = 16, kRowThreads = 64 * kRows, kLanes = kRowThreads / (kRows / 4);
template <int kEach> __global__ __launch_bounds__(kRowThreads) void k_distill_rows(DistillArgs a) {
  __shared__ float sh[kLanes * (kRows + 1)];
  __shared__ double parts[kRowThreads / 64][kDistillSums];
  const int nvalid = valid_rows(a.n_scored, a.chunk_start, a.chunk_rows), r0 = blockIdx.x * kRows;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  double q[kDistillSums] = {};
  if (r0 < nvalid) {
    // what the wave's row needs is under way before the partial sums are
    const int64_t r = r0 + wave, ci = a.chunk_start + (r < nvalid ? r : nvalid - 1), slot = a.row_index[ci];
    const float zt = a.zt[ci], w = weight_of(a, slot);
    Alternatives<kEach> alt;
    alt.load(a, slot);
    float z[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int j = 64 * e + lane;
      z[e] = a.zk[(ci - a.chunk_start) * a.k + (j < a.k ? j : 0)];
    }
    // a thread adds every kLanes-th partial of four rows; the rows behind the valid ones hold whatever the buffer held
    const int quad = threadIdx.x & 3, part = threadIdx.x >> 2;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = part; i < a.n_partials; i += kLanes) {
      const float4 x = *reinterpret_cast<const float4*>(a.part_sum + (int64_t)i * a.chunk_rows + r0 + quad * 4);
      s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
    }
    float* const cell = sh + part * (kRows + 1) + quad * 4;
    cell[0] = s.x; cell[1] = s.y; cell[2] = s.z; cell[3] = s.w;
    __syncthreads();
    if (r < nvalid) {
      float S = 0.f;
#pragma unroll
      for (int i = 0; i < kLanes / 64; ++i) S += sh[(64 * i + lane) * (kRows + 1) + wave];
      S = lanes_sum<64>(S);
      const float c2 = fmaf(zt, a.scale2, kStashMargin2);
      alt.weigh(a, alt.best_t());
      const double log2_sum = (double)c2 + log2((double)S);        // of exponentials in the log2 domain, with the very c2 that the launch took
      double kl = 0.0;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        if (alt.q[e] != 0.0) kl += alt.q[e] * (alt.log_q[e] - ((double)z[e] * (double)a.scale2 - log2_sum) * LN2);
      }
      kl = wave_sum(kl);
      // the alternative that the student thinks most of is beyond the operands' range: not in the loss, as an empty row
      // (NaN is not: the launches' clamps go past it, so it enters the gradients with the row's scale)
      const bool number = fabs(kl) < (double)INFINITY;
      const bool saturated = number && ((double)zt * (double)a.scale2 - log2_sum) * LN2 < (double)kSaturatedLogp;
      if (lane == 0) a.out_kl[slot] = (float)kl;
      if (saturated) q[1] += 1.0; else q[0] += (double)w * kl;
      q[2] += alt.too_large;
      if (a.row_scale != nullptr && saturated && lane == 0) a.row_scale[ci] = 0.f;
      if (a.row_scale != nullptr && !saturated) {
        uint16_t* const row = a.estash + r * a.lde;
        // The row's scale.  Of a small mass beside a large sum (S is 2^-60 over the probability of the student's likeliest alternative, 2^80 at most) it is less than floats
        // hold, though the gradient is not: the stored row is brought to a sum from 1 to 2 then, by a power of two.  (Alternatives that both hold for impossible: rare.)
        float down = 1.f;
        double scale = (double)w * (double)a.temperature * alt.m / (double)S;
        if (__builtin_expect(fabs(scale) < kLeastScale && scale != 0.0 && S > 1.f, 0)) {
          down = ldexpf(1.f, -ilogbf(S));
          scale /= (double)down;
#pragma unroll 1
          for (int v = lane * 8; v < a.V; v += 512) {  // (rows are padded to whole vectors)
            u32x4 x = *reinterpret_cast<const u32x4*>(row + v);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = pack_bf16(bf16_low(x[i]) * down, bf16_high(x[i]) * down);
            *reinterpret_cast<u32x4*>(row + v) = x;
          }
          __threadfence_block();                       // (the places below are other lanes' here)
        }
        if (lane == 0) a.row_scale[ci] = number ? (float)scale : __builtin_nanf("");
        float share[kEach];
        bool first[kEach];
        alt.by_id(a.k, share, first);
#pragma unroll
        for (int e = 0; e < kEach; ++e)
          if (first[e]) {
            const float x = down * __builtin_amdgcn_exp2f(fminf(fmaf(z[e], a.scale2, -c2), kStashClamp2)) - down * S * share[e];
            row[alt.id[e]] = (uint16_t)pack_bf16(x, 0.f);
          }
      }
    }
  }
  if (lane == 0) {
#pragma unroll
    for (int k = 0; k < kDistillSums; ++k) parts[wave][k] = q[k];
  }
  __syncthreads();
  if (threadIdx.x < kDistillSums) {
    double t = 0.0;
    for (int w = 0; w < kRowThreads / 64; ++w) t += parts[w][threadIdx.x];
    a.loss_partials[(a.partial_block_offset + blockIdx.x) * kDistillSums + threadIdx.x] = t;
  }
}

// ----------------------------------------------------------------------------
// fp32: a wave per row of the materialised logits, which become dz.  Up to 64 kHeld logits stay in registers between the three looks at them.
// ----------------------------------------------------------------------------
template <int kEach, int kHeld> __global__ __launch_bounds__(256) void k_distill_f32(DistillArgs a) {
  __shared__ double parts[4][kDistillSums];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.x * 4 + wave;
  double q[kDistillSums] = {};
  if (r < valid_rows(a.n_scored, a.chunk_start, a.chunk_rows)) {
    const int64_t slot = a.row_index[a.chunk_start + r];
    float* const row = a.Z + (int64_t)r * a.ldz;
    const float w = weight_of(a, slot), inv_T = 1.f / a.temperature;
    Alternatives<kEach> alt;
    alt.load(a, slot);
    float z[kEach], held[kHeld > 0 ? kHeld : 1];
#pragma unroll
    for (int e = 0; e < kEach; ++e) z[e] = alt.id[e] >= 0 ? row[alt.id[e]] : 0.f;
    // f(place in registers, id) for the lane's logits
    auto each = [&](auto f) {
      if constexpr (kHeld > 0) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
          if (i * 64 < a.V && i * 64 + lane < a.V) f(held[i], i * 64 + lane);
      } else {
        for (int v = lane; v < a.V; v += 64) { held[0] = row[v]; f(held[0], v); }
      }
    };
    float mx = -INFINITY;
    each([&](float& x, int v) { if (kHeld > 0) x = row[v]; mx = fmaxf(mx, x); });
    mx = wave_max(mx);
    float s = 0.f;
    each([&](float& x, int) { const float e = expf((x - mx) * inv_T); if (kHeld > 0) x = e; s += e; });
    const float S = lanes_sum<64>(s);
    const double log_S = log((double)S);
    alt.weigh(a, alt.best_t());
    double kl = 0.0;
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (alt.q[e] != 0.0) kl += alt.q[e] * (alt.log_q[e] - (((double)z[e] - (double)mx) / (double)a.temperature - log_S));
    kl = wave_sum(kl);
    if (lane == 0) a.out_kl[slot] = (float)kl;
    q[0] = (double)w * kl;
    q[2] = alt.too_large;
    if (a.write_dz) {
      const double g = (double)w * (double)a.temperature * alt.m;
      const float scale = (float)(g / (double)S);
      float share[kEach];
      bool first[kEach];
      alt.by_id(a.k, share, first);
      each([&](float& x, int v) { row[v] = scale * (kHeld > 0 ? x : expf((x - mx) * inv_T)); });
      __threadfence_block();                           // (the places below are other lanes' above)
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (first[e]) row[alt.id[e]] = scale * expf((z[e] - mx) * inv_T) - (float)g * share[e];
    }
  }
  if (lane == 0) {
#pragma unroll
    for (int k = 0; k < kDistillSums; ++k) parts[wave][k] = q[k];
  }
  __syncthreads();
  if (threadIdx.x < kDistillSums)
    a.loss_partials[(a.partial_block_offset + blockIdx.x) * kDistillSums + threadIdx.x] =
        (parts[0][threadIdx.x] + parts[1][threadIdx.x]) + (parts[2][threadIdx.x] + parts[3][threadIdx.x]);
}

constexpr int FINAL_THREADS = 256;
__global__ __launch_bounds__(FINAL_THREADS) void k_distill_final(const double* parts, int64_t blocks, const int64_t* n_scored, const int64_t* n_empty,
                                                                 double scale, double* out_d, int64_t* out_i) {
  __shared__ double sh[FINAL_THREADS / 64][kDistillSums];
  double q[kDistillSums] = {};
  for (int64_t b = threadIdx.x; b < blocks; b += FINAL_THREADS)
#pragma unroll
    for (int k = 0; k < kDistillSums; ++k) q[k] += parts[b * kDistillSums + k];
#pragma unroll
  for (int k = 0; k < kDistillSums; ++k) {
    q[k] = wave_sum(q[k]);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6][k] = q[k];
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
#pragma unroll
  for (int k = 0; k < kDistillSums; ++k) q[k] = (sh[0][k] + sh[1][k]) + (sh[2][k] + sh[3][k]);
  *out_d = scale * q[0];
  out_i[0] = *n_scored;
  out_i[1] = *n_empty;
  out_i[2] = (int64_t)(q[1] + 0.5);
  out_i[3] = (int64_t)(q[2] + 0.5);
}

__global__ __launch_bounds__(256) void k_to_bf16(const float* in, uint16_t* out, int64_t n) {
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8; i < n; i += (int64_t)gridDim.x * 256 * 8) {
    const u32x4 lo = load_any<4, u32x4>(in + i), hi = load_any<4, u32x4>(in + i + 4);
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      w[e] = pack_bf16(__uint_as_float(lo[2 * e]), __uint_as_float(lo[2 * e + 1]));
      w[2 + e] = pack_bf16(__uint_as_float(hi[2 * e]), __uint_as_float(hi[2 * e + 1]));
    }
    store_any<2>(out + i, w);
  }
}

}  // namespace

// Alternatives of a lane: as few as do (a double exponential each).
template <class F> static F by_count(int k, F one, F two, F four) { return k <= 64 ? one : k <= 128 ? two : four; }
static_assert(kMostAlternatives <= 256, "four to a lane");

void launch_distill_targets(const DistillArgs& a, hipStream_t stream) {
  const int64_t blocks = (a.N + 3) / 4, wide = blocks < (1 << 21) ? blocks : 1 << 21;
  hipLaunchKernelGGL(by_count(a.k, k_distill_targets<1>, k_distill_targets<2>, k_distill_targets<4>), dim3((unsigned)wide, (unsigned)((blocks + wide - 1) / wide)),
                     dim3(256), 0, stream, a);
}
void launch_distill_logits(const DistillArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(k_distill_logits, dim3(a.chunk_rows), dim3(256), 0, stream, a);
}
void launch_distill_hidden_nan(const DistillArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(k_distill_hidden_nan, dim3((a.V + kPartialRows - 1) / kPartialRows), dim3(256), 0, stream, a);
}
void launch_distill_rows(const DistillArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(by_count(a.k, k_distill_rows<1>, k_distill_rows<2>, k_distill_rows<4>), dim3(a.chunk_rows / kRows), dim3(kRowThreads), 0, stream, a);
}
int distill_row_blocks(int chunk_rows) { return chunk_rows / kRows; }
int distill_f32_blocks(int64_t rows) { return (int)((rows + 3) / 4); }
// Rows of up to 512 logits stay in registers, eight to a lane (call, d = 64, k = 16, us, so and with every look from memory: 256 rows, V = 64 28.3 and 28.2, 300 30.2 and 30.9,
// 512 32.4 and 33.7; 2048 rows of 512 69.0 and 69.7).  Sixteen to a lane would do the same for longer ones (256 rows, V = 1000 40.0 for 43.1) and cost a little here (64 rows, V = 512 30.8 and 31.3).
void launch_distill_f32(const DistillArgs& a, int rows, hipStream_t stream) {
  const auto kernel = a.V <= 8 * 64 ? by_count(a.k, k_distill_f32<1, 8>, k_distill_f32<2, 8>, k_distill_f32<4, 8>)
                                    : by_count(a.k, k_distill_f32<1, 0>, k_distill_f32<2, 0>, k_distill_f32<4, 0>);
  hipLaunchKernelGGL(kernel, dim3(distill_f32_blocks(rows)), dim3(256), 0, stream, a);
}
void launch_distill_final(const double* parts, int64_t blocks, const int64_t* n_scored, const int64_t* n_empty, double scale, double* out_d, int64_t* out_i,
                          hipStream_t stream) {
  hipLaunchKernelGGL(k_distill_final, dim3(1), dim3(FINAL_THREADS), 0, stream, parts, blocks, n_scored, n_empty, scale, out_d, out_i);
}
void launch_to_bf16(const float* in, void* out, int64_t n, hipStream_t stream) {
  const int64_t blocks = (n / 8 + 255) / 256;
  hipLaunchKernelGGL(k_to_bf16, dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, stream, in, static_cast<uint16_t*>(out), n);
}

}  // namespace mrl
