// Top alternatives of given logits, with the log-probs of given tokens and the entropy.  Row n of [N, V], s2 = log2(e) / T:
//   u_v = z_v s2 - m s2,  S = sum 2^u,  E = sum 2^u u     (m: the largest logit met; all in the log2 domain)
//   lse = (m s2 + log2 S) ln 2,  entropy = (log2 S - E / S) ln 2,  log-prob = (z s2 - m s2 - log2 S) ln 2
//   alternatives: the k largest by (logit, then the lower id first), exactly those
// One pass reads the logits once.  A thread notes the largest of every few tiles it has seen.  The k-th largest of the threads' maxima is a lower bound of the
// k-th largest logit (each maximum is another element); behind the pass, the notes that reach it say where the logits that do can be, and those places, k and a
// little, are read again: what reaches the bound goes to a list in LDS, which is sorted.  So the pass itself has no branch, barrier or atomic for the alternatives' sake.
// (With a list kept during the pass, under a bound renewed behind tiles 0, 1, 3, 7 ..., the entries' branches and atomics took as long as a third of the pass: 4096 rows of
// 151936 in bf16, k = 64 264 us, now 229; 620 rows of 50257 floats 36 and 30.)  Where the list is too long (sorted or constant rows), and for rows with
// NaN, the workgroup selects by digits of the whole key instead, in at most seven further passes.
// Few rows are split over several workgroups each, whose lists and sums a second launch joins: a launch in which the last of them to end joins them would need
// counters that are zero before the call.
// Memory bounds it in 32 bits (4096 rows of 151936: k = 64 428 us, 5.8 TB/s; k = 0 408, 6.1), and the vector unit all but does in 16 (229 us, 5.4 TB/s): 9.5 issue slots a
// logit, four of them the exponential's.
#include "../../include/mrl.h"
#include "mrl_internal.h"
#include "mrl_vec.h"

namespace mrl {
namespace {

constexpr int kMostThreads = 512;                      // of a workgroup
constexpr int kWavesAtOnce = 8;                        // per SIMD: four workgroups to a compute unit
constexpr int kPer = 16;                               // logits of a thread in a tile
constexpr int kMostTop = 256;                          // alternatives of a call at most (the bound needs as many threads)
constexpr int kHeld = 8;                               // entries that the list has room for, per thread
constexpr int kMostList = 1024;                        // entries of a list that is sorted (k and a little as a rule): every entry is compared with every other
constexpr int kNotes = 32;                             // of a thread, each the largest of as many tiles as that makes (one up to V = 262144)
constexpr int kPairs = 512;                            // notes that reach the bound, at most (about 350 where 256 alternatives are asked for)
constexpr int kMostSplit = 256;
constexpr int kIdBits = 24;                            // V <= 2^24
constexpr uint64_t kIdMask = ((uint64_t)1 << kIdBits) - 1;
constexpr float kNone = -1e30f;                        // the running maximum of no logits: finite, and so is its product with s2
constexpr float kLeastU = -200.f;                      // 2^u is 0 there; u itself must not be infinite in the product 2^u u
constexpr float kLeastSum = 0x1p-100f;                 // of a row: its largest logit is 2^u with u the rounding of m s2, less than -100 only beyond 1e9
constexpr double LN2 = 0.6931471805599453;

struct Part { float m2, S, E; };
struct TopArgs {
  const void* z; int64_t ld; const int32_t* targets; const uint8_t* mask;
  int64_t N; int V, k, split, slice;
  float s2;
  int32_t* ids; float* top; float* logp; float* lse; float* entropy;
  Part* parts; uint64_t* keys;                         // [N][split], [N][split][k]
};

// Order of the logits as whole numbers: NaN above everything, zeros of either sign alike, no number is 0.
__device__ inline uint32_t ordered(float z) {
  const uint32_t b = __float_as_uint(z + 0.f);
  return z != z ? ~0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float from_ordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ inline uint64_t key_of(float z, int id) { return (uint64_t)ordered(z) << kIdBits | (kIdMask - (uint64_t)id); }
__device__ inline int id_of(uint64_t key) { return (int)(kIdMask - (key & kIdMask)); }
__device__ inline float logit_of(uint64_t key) { return from_ordered((uint32_t)(key >> kIdBits)); }

template <bool kBf16> __device__ inline float logit_at(const void* row, int v) {
  return kBf16 ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(row)[v] << 16) : static_cast<const float*>(row)[v];
}

// What a thread of a workgroup of T looks at of a tile: vectors of 16 bytes, T apart.  Behind `end` it finds -infinity.
template <bool kBf16, int T> struct Tile {
  static constexpr int kVec = kBf16 ? 8 : 4, kLoads = kPer / kVec, kSize = kBf16 ? 2 : 4, kLogits = T * kPer;
  u32x4 w[kLoads];
  __device__ static int id(int at, int i) { return at + (i / kVec * T + (int)threadIdx.x) * kVec + i % kVec; }
  __device__ void load(const void* row, int at, int end) {
    if (at + kLogits <= end) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) w[j] = load_any<kSize, u32x4>(static_cast<const char*>(row) + (int64_t)id(at, j * kVec) * kSize);
      return;
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j) w[j] = load_to(row, id(at, j * kVec), end);
  }
  // The vector from logit v on, -infinity from `end` on.
  __device__ static u32x4 load_to(const void* row, int v, int end) {
    if (v + kVec <= end) return load_any<kSize, u32x4>(static_cast<const char*>(row) + (int64_t)v * kSize);
    const uint32_t none = kBf16 ? 0xff80ff80u : 0xff800000u;
    u32x4 w = {none, none, none, none};
#pragma unroll
    for (int e = 0; e < kVec - 1; ++e)
      if (v + e < end) {
        if (kBf16) {
          const uint32_t b = static_cast<const uint16_t*>(row)[v + e];
          w[e >> 1] = e & 1 ? (w[e >> 1] & 0xffffu) | b << 16 : (w[e >> 1] & 0xffff0000u) | b;
        } else {
          w[e] = static_cast<const uint32_t*>(row)[v + e];
        }
      }
    return w;
  }
  __device__ float operator[](int i) const {
    if (kBf16) return i & 1 ? bf16_high(w[i / 8][i % 8 / 2]) : bf16_low(w[i / 8][i % 8 / 2]);
    return __uint_as_float(w[i / 4][i % 4]);
  }
};

template <bool kBf16, int T> __device__ inline void load_vector(const void* row, int v, int end, float (&z)[Tile<kBf16, T>::kVec]) {
  const u32x4 w = Tile<kBf16, T>::load_to(row, v, end);
#pragma unroll
  for (int e = 0; e < Tile<kBf16, T>::kVec; ++e)
    z[e] = kBf16 ? e & 1 ? bf16_high(w[e >> 1]) : bf16_low(w[e >> 1]) : __uint_as_float(w[e & 3]);
}

template <int T> struct Shared {
  static constexpr int kWaves = T / 64, kKeys = kHeld * T;
  union {
    uint16_t notes[kNotes][T];                         // upper half of the ordered number, as many bits as the bound has
    uint64_t keys[kKeys];                              // the list
  };
  union {
    uint64_t best[kMostTop];
    uint32_t pairs[kPairs];
  };
  uint32_t maxima[T];
  float wave[kWaves][4];
  uint32_t scan[kWaves];
  uint32_t n_pairs, count /*entries of the list*/, bound, digit, above, inside;
};

// A lower bound of the k-th largest of the threads' numbers sh.maxima, exact in its upper kBoundBits bits, by bisection in the first wave.  0: fewer than k
// are above 0.  Ends with a barrier.
constexpr int kBoundBits = 16;                         // (as many as a note has)
template <int T> __device__ inline void find_bound(Shared<T>& sh, int k) {
  constexpr int kWaves = T / 64;
  __syncthreads();
  if (threadIdx.x < 64) {
    uint32_t m[kWaves], t = 0;
#pragma unroll
    for (int j = 0; j < kWaves; ++j) m[j] = sh.maxima[j * 64 + threadIdx.x];
    for (int bit = 31; bit > 31 - kBoundBits; --bit) {
      const uint32_t c = t | 1u << bit;
      int n = 0;
#pragma unroll
      for (int j = 0; j < kWaves; ++j) n += __popcll(__ballot(m[j] >= c));
      if (n >= k) t = c;
    }
    if (threadIdx.x == 0) sh.bound = t;
  }
  __syncthreads();
}

// The k largest of the list's sh.count keys, largest first, to sh.best (zeros where there are fewer).  Begins behind a barrier.
template <int T> __device__ inline void sort_best(Shared<T>& sh, int k) {
  int n = (int)sh.count;
  if (n > 2 * k + 64) {
    // fewer of them: those that reach the k-th largest of the threads' maxima
    uint64_t own[kHeld];
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int i = j * T + threadIdx.x;
      own[j] = i < n ? sh.keys[i] : 0;
      most = larger(most, (uint32_t)(own[j] >> kIdBits));
    }
    sh.maxima[threadIdx.x] = most;
    find_bound(sh, k);                                 // (its first barrier: all keys have been read)
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    const uint32_t bound = sh.bound;
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (own[j] != 0 && (uint32_t)(own[j] >> kIdBits) >= bound) sh.keys[atomicAdd(&sh.count, 1u)] = own[j];
    __syncthreads();
    n = (int)sh.count;
  }
  // a key's place is the number of larger ones: no two are alike (but for the zeros that stand for none)
  for (int i = threadIdx.x; i < n; i += T) {
    const uint64_t key = sh.keys[i];
    int place = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) place += sh.keys[j] > key;
    if (place < k) sh.best[place] = key;
  }
  for (int i = n + threadIdx.x; i < k; i += T) sh.best[i] = 0;
  __syncthreads();
}

// The list by digits of the whole key, whatever the logits are: at most 2 k + 64 entries, the k largest of logits begin .. end - 1 among them.
template <bool kBf16, int T> __device__ inline void collect_by_digits(Shared<T>& sh, const void* row, int begin, int end, int k) {
  constexpr int kBits = T == 512 ? 12 : 10, kBins = 1 << kBits;           // eight bins to a thread
  static_assert(kBins == 8 * T && kBins * 4 <= Shared<T>::kKeys * 8, "the bins take the list's place");
  uint32_t* const hist = reinterpret_cast<uint32_t*>(sh.keys);
  uint64_t prefix = 0;
  uint32_t above = 0;                                  // keys above the prefix: fewer than k
  int rest = 32 + kIdBits;                             // bits below the prefix
#pragma unroll 1                                       // (rare: registers count for more than its loops' speed)
  for (;;) {
    const int bits = rest < kBits ? rest : kBits, shift = rest - bits;
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += T) hist[i] = 0;
    __syncthreads();
#pragma unroll 1
    for (int v = begin + threadIdx.x; v < end; v += T) {
      const uint64_t key = key_of(logit_at<kBf16>(row, v), v);
      if (key >> rest == prefix) atomicAdd(&hist[(key >> shift) & ((1u << bits) - 1)], 1u);
    }
    __syncthreads();
    // from the highest digit down, eight to a thread: the one that holds the (k - above)-th key
    const int first = kBins - 8 * (int)(threadIdx.x + 1);
    uint32_t sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += hist[first + i];
    uint32_t incl = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const uint32_t up = __shfl_up(incl, off);
      if ((int)(threadIdx.x & 63) >= off) incl += up;
    }
    if ((threadIdx.x & 63) == 63) sh.scan[threadIdx.x >> 6] = incl;
    __syncthreads();
    for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) incl += sh.scan[w];
    const uint32_t need = (uint32_t)k - above;
    if (incl - sum < need && need <= incl) {
      uint32_t run = incl - sum;
      int i = 7;
      while (run + hist[first + i] < need) { run += hist[first + i]; --i; }
      sh.digit = first + i; sh.above = run; sh.inside = hist[first + i];
    }
    __syncthreads();
    prefix = prefix << bits | sh.digit;
    above += sh.above;
    rest = shift;
    if (above + sh.inside <= 2u * k + 64) break;       // (behind the last digit a single key is inside)
  }
  const uint64_t least = prefix << rest;
  __syncthreads();
  if (threadIdx.x == 0) sh.count = 0;
  __syncthreads();
#pragma unroll 1
  for (int v = begin + threadIdx.x; v < end; v += T) {
    const uint64_t key = key_of(logit_at<kBf16>(row, v), v);
    if (key >= least) sh.keys[atomicAdd(&sh.count, 1u)] = key;
  }
  __syncthreads();
}

// All threads' sums as one, relative to the largest of their m2, in a fixed order; known to all.  (A part without logits has S = 0 and the least m2.)
template <int kLanes> __device__ inline Part join_lanes(Part p) {
  const float m2 = over_lanes<kLanes>(p.m2, [](float a, float b) { return fmaxf(a, b); }), d = p.m2 - m2, c = __builtin_amdgcn_exp2f(d);
  return {m2, lanes_sum<kLanes>(c * p.S), lanes_sum<kLanes>(c * fmaf(p.S, d, p.E))};
}
template <int T> __device__ inline Part join_all(Shared<T>& sh, Part p) {
  p = join_lanes<64>(p);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) { float* w = sh.wave[threadIdx.x >> 6]; w[0] = p.m2; w[1] = p.S; w[2] = p.E; }
  __syncthreads();
  const int w = threadIdx.x & 7;                       // (eight lanes join them, of waves that there are not nothing)
  return join_lanes<8>(w < T / 64 ? Part{sh.wave[w][0], sh.wave[w][1], sh.wave[w][2]} : Part{p.m2, 0.f, 0.f});
}

// Sums of a row that the pass has none for: its largest logit is NaN, infinite, below kNone, or so large that m s2, its distance from kNone s2, or 2 to the power of its rounding is not finite
// (there E alone may be NaN).  Two passes, the differences to the largest logit first.  S is NaN where there is no distribution.
template <bool kBf16, int T> __device__ inline void careful_sums(Shared<T>& sh, const TopArgs& a, const void* row, double& offset, float& S, float& E) {
  uint32_t most = 0;
#pragma unroll 1
  for (int v = threadIdx.x; v < a.V; v += T) most = larger(most, ordered(logit_at<kBf16>(row, v)));
  most = lanes_max<64>(most);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.scan[threadIdx.x >> 6] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < T / 64; ++w) most = larger(most, sh.scan[w]);
  const float m = from_ordered(most);
  offset = 0; S = __builtin_nanf(""); E = 0.f;
  if (!(fabsf(m) < INFINITY)) return;
  Part p = {0.f, 0.f, 0.f};
#pragma unroll 1
  for (int v = threadIdx.x; v < a.V; v += T) {
    const float u = (logit_at<kBf16>(row, v) - m) * a.s2, e = __builtin_amdgcn_exp2f(u);
    p.S += e;
    p.E = fmaf(e, fmaxf(u, kLeastU), p.E);
  }
  p = join_all(sh, p);
  offset = (double)m * (double)a.s2; S = p.S; E = p.E;
}

// A row's outputs: sums in p, the alternatives in sh.best.
template <bool kBf16, int T> __device__ inline void put_row(Shared<T>& sh, const TopArgs& a, int64_t n, const Part& p) {
  const void* row = static_cast<const char*>(a.z) + n * a.ld * (kBf16 ? 2 : 4);
  double offset = p.m2;
  float S = p.S, E = p.E;
  if (!(S > kLeastSum && S < INFINITY) || E != E) careful_sums<kBf16>(sh, a, row, offset, S, E);
  if ((int)(threadIdx.x & ~63u) >= (a.k > 1 ? a.k : 1)) return;      // (waves without outputs; no barrier from here on)
  const double log2_S = log2((double)S);
  // As the sums took it: the difference to the offset is exact, so that far from zero (rows masked throughout with the type's lowest value) the log-probs are those of the
  // logits' differences.  z / T - lse was off by what the scale's rounding makes of z itself.
  const auto log_prob = [&](float z) { return (float)(((double)z * (double)a.s2 - offset - log2_S) * LN2); };
  for (int i = threadIdx.x; i < a.k; i += T) {
    const uint64_t key = sh.best[i];
    if (a.ids != nullptr) a.ids[n * a.k + i] = id_of(key);
    if (a.top != nullptr) a.top[n * a.k + i] = log_prob(logit_of(key));
  }
  if (threadIdx.x == 0) {
    if (a.lse != nullptr) a.lse[n] = (float)((offset + log2_S) * LN2);
    if (a.entropy != nullptr) a.entropy[n] = (float)((log2_S - (double)E / (double)S) * LN2);
    if (a.logp != nullptr) {
      const int y = a.targets[n];
      a.logp[n] = y >= 0 && y < a.V ? log_prob(logit_at<kBf16>(row, y)) : 0.f;
    }
  }
}

template <int T> __device__ inline void put_masked_row(const TopArgs& a, int64_t n) {
  for (int i = threadIdx.x; i < a.k; i += T) {
    if (a.ids != nullptr) a.ids[n * a.k + i] = -1;
    if (a.top != nullptr) a.top[n * a.k + i] = 0.f;
  }
  if (threadIdx.x == 0) {
    if (a.lse != nullptr) a.lse[n] = 0.f;
    if (a.entropy != nullptr) a.entropy[n] = 0.f;
    if (a.logp != nullptr) a.logp[n] = 0.f;
  }
}

template <bool kBf16, int T> __global__ __launch_bounds__(T, kWavesAtOnce) void k_top(TopArgs a) {
  using Tile = Tile<kBf16, T>;
  constexpr int kTileLogits = Tile::kLogits;
  static_assert(kMostList <= Shared<T>::kKeys && 2 * kMostTop + 64 <= kMostList, "lists have their room");
  __shared__ Shared<T> sh;
  const int64_t item = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, n = item / a.split;
  if (n >= a.N) return;
  if (a.mask != nullptr && a.mask[n] == 0) {
    if (a.split == 1) put_masked_row<T>(a, n);
    return;
  }
  const int part = (int)(item - n * a.split), begin = part * a.slice, end = a.V - begin < a.slice ? a.V : begin + a.slice;
  const void* row = static_cast<const char*>(a.z) + n * a.ld * (kBf16 ? 2 : 4);
  const int k = a.k < end - begin ? a.k : end - begin;
  const int tiles = (end - begin + kTileLogits - 1) / kTileLogits, per_note = (tiles + kNotes - 1) / kNotes;
  if (threadIdx.x == 0) sh.n_pairs = sh.count = 0;
  float m = kNone, m2 = kNone * a.s2, S = 0.f, E = 0.f, note = -INFINITY;
  Tile next;
  next.load(row, begin, end);
  int left = per_note, notes = 0;                      // tiles of the note under way, notes so far
  for (int tile = 0; tile < tiles; ++tile) {
    const Tile z = next;
    if (tile + 1 < tiles) next.load(row, begin + (tile + 1) * kTileLogits, end);
    float most = z[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) most = fmaxf(most, z[i]);
    if (most > m) {
      const float to = most * a.s2, d = m2 - to, c = __builtin_amdgcn_exp2f(d);
      E = c * fmaf(S, d, E);
      S = c * S;
      m = most; m2 = to;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float u = fmaf(z[i], a.s2, -m2), e = __builtin_amdgcn_exp2f(u);
      S += e;
      E = fmaf(e, fmaxf(u, kLeastU), E);
    }
    note = fmaxf(note, most);
    if (--left == 0 || tile + 1 == tiles) { sh.notes[notes++][threadIdx.x] = (uint16_t)(ordered(note) >> 16); note = -INFINITY; left = per_note; }
  }
  sh.maxima[threadIdx.x] = m > kNone ? ordered(m) : 0;
  const Part p = join_all(sh, {m2, S, E});
  if (k > 0) {
    find_bound(sh, k);
    const float bound = sh.bound == 0 ? -INFINITY : from_ordered(sh.bound);
    for (int i = 0; i < notes; ++i)
      if (sh.notes[i][threadIdx.x] >= sh.bound >> 16) {
        const uint32_t at = atomicAdd(&sh.n_pairs, 1u);
        if (at < (uint32_t)kPairs) sh.pairs[at] = (uint32_t)i << 16 | threadIdx.x;
      }
    __syncthreads();
    const uint32_t n_pairs = sh.n_pairs;
    if (n_pairs <= (uint32_t)kPairs) {
      // a vector of a noted tile per thread and step
      constexpr int kVec = Tile::kVec, kLoads = Tile::kLoads;
      const int each = per_note * kLoads;
      for (int q = threadIdx.x; q < (int)n_pairs * each; q += T) {
        const int which = q / each, in = q - which * each, thread = (int)(sh.pairs[which] & 0xffffu);
        const int tile = (int)(sh.pairs[which] >> 16) * per_note + in / kLoads;
        const int v = begin + tile * kTileLogits + (in % kLoads * T + thread) * kVec;
        if (tile >= tiles || v >= end) continue;
        float z[kVec];
        load_vector<kBf16, T>(row, v, end, z);
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (!(z[e] < bound) && v + e < end) {
            const uint32_t place = atomicAdd(&sh.count, 1u);
            if (place < (uint32_t)kMostList) sh.keys[place] = key_of(z[e], v + e);
          }
      }
    }
    __syncthreads();
    // (a NaN is the only thing that makes S one, but for an infinite logit: the comparisons above went past it)
    if (n_pairs > (uint32_t)kPairs || sh.count > (uint32_t)kMostList || p.S != p.S) collect_by_digits<kBf16>(sh, row, begin, end, k);
    sort_best(sh, k);
  }
  if (a.split == 1) {
    put_row<kBf16>(sh, a, n, p);
    return;
  }
  if (threadIdx.x == 0) a.parts[item] = p;
  // (a last slice may be shorter than the list: zeros, which stand for none, where it has no logits)
  for (int i = threadIdx.x; i < a.k; i += T) a.keys[item * a.k + i] = i < k ? sh.best[i] : 0;
}

template <bool kBf16> __global__ __launch_bounds__(kMostThreads) void k_top_join(TopArgs a) {
  constexpr int T = kMostThreads;
  __shared__ Shared<T> sh;
  const int64_t n = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (n >= a.N) return;
  if (a.mask != nullptr && a.mask[n] == 0) { put_masked_row<T>(a, n); return; }
  const int count = a.split * a.k;                     // (at most kKeys)
  for (int i = threadIdx.x; i < count; i += T) sh.keys[i] = a.keys[n * count + i];
  if (threadIdx.x == 0) sh.count = (uint32_t)count;
  const Part p = join_all(sh, (int)threadIdx.x < a.split ? a.parts[n * a.split + threadIdx.x] : Part{kNone * a.s2, 0.f, 0.f});
  if (a.k > 0) sort_best(sh, a.k);
  put_row<kBf16>(sh, a, n, p);
}

// Workgroups of a row: one where there are rows enough for the chip (four workgroups to a compute unit), else as many as it has room for, each with a
// quarter of a tile or more.  The join takes longer the more keys it is given, so that their lists hold 1024 together where that leaves no more than two tiles to each
// (one row of 151936 floats, us, with 4096 and 1024: k = 64 20.2 and 16.6; 48 rows of 128256, k = 200 30.1 and 24.0), and at most what the join's list holds.
struct Split { int split, slice; };
Split split_of(int64_t N, int V, int k) {
  constexpr int kTileLogits = kMostThreads * kPer, kMostKeys = Shared<kMostThreads>::kKeys;
  int64_t s = N > 0 ? 1024 / N : 1;
  if (s > kMostSplit) s = kMostSplit;
  if (k > 0) {
    const int64_t few = 1024 / k, by_tiles = V / (2 * kTileLogits), most = few > by_tiles ? few : by_tiles;
    if (s > most) s = most;
    if (s > kMostKeys / k) s = kMostKeys / k;
  }
  const int64_t by_length = (V + kTileLogits / 4 - 1) / (kTileLogits / 4);
  if (s > by_length) s = by_length;
  if (s <= 1) return {1, V};
  const int slice = (int)round_up((V + s - 1) / s, 64);
  return {(V + slice - 1) / slice, slice};
}

// Workgroups of 128 where a row is short: what a row costs beyond its logits is the same latencies with any number of threads, and eight such rows are under way where
// two of 512 were (16384 rows, us: of 1000 floats, k = 10 111 and 37, of 9000 in bf16 146 and 75, of 37000 262 and 243; of 151936 in bf16, k = 64 (4096 rows) 231 and 295).
// With more alternatives the bound by the threads' maxima is too wide.
constexpr int kFewThreads = 128;
bool short_rows(int split, int V, int k) { return split == 1 && ((V <= 65536 && k <= kFewThreads / 4) || (V <= 32768 && k <= kFewThreads / 2)); }

constexpr int64_t kMostRows = (int64_t)1 << 30, kMostWide = 1 << 21;
dim3 grid_of(int64_t groups) {
  const int64_t wide = groups < kMostWide ? groups : kMostWide;
  return dim3((unsigned)wide, (unsigned)((groups + wide - 1) / wide));
}
bool top_shape(int64_t N, int32_t V, int32_t k) { return N >= 0 && N <= kMostRows && V > 0 && V <= 1 << kIdBits && k >= 0 && k <= kMostTop && k <= V; }
bool is_float_type(int32_t t) { return t == MRL_F32 || t == MRL_BF16; }
size_t parts_bytes(int64_t N, int split) { return (size_t)round_up(N * split * (int64_t)sizeof(Part), 256); }

}  // namespace
}  // namespace mrl

using namespace mrl;

extern "C" size_t mrl_top_logprobs_workspace(int64_t N, int32_t V, int32_t k) {
  if (!top_shape(N, V, k)) return 0;
  const Split s = split_of(N, V, k);
  return s.split == 1 ? 256 : parts_bytes(N, s.split) + (size_t)round_up(N * s.split * k * 8, 256);
}

extern "C" int mrl_top_logprobs(const void* logits, int64_t row_stride, const int32_t* target_ids, const uint8_t* token_mask, int64_t N, int32_t V,
                                int32_t k, int32_t dtype, float temperature, int32_t* out_ids, float* out_top_logp, float* out_logp, float* out_lse,
                                float* out_entropy, void* workspace, size_t workspace_bytes, void* stream) {
  if (!is_float_type(dtype)) return MRL_ERR_DTYPE;
  if (!top_shape(N, V, k) || row_stride < V || row_stride > ((int64_t)1 << 40)) return MRL_ERR_SHAPE;
  if (!(temperature >= 1e-4f && temperature <= 1e4f)) return MRL_ERR_CONFIG;
  if (N == 0) return MRL_OK;
  if (!logits || (k > 0 && !out_ids && !out_top_logp) || (out_logp && !target_ids) || (k == 0 && !out_logp && !out_lse && !out_entropy)) return MRL_ERR_NULL;
  const Split s = split_of(N, V, k);
  if (s.split > 1 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < mrl_top_logprobs_workspace(N, V, k)))
    return MRL_ERR_WORKSPACE;
  const int rc = require_gfx950();
  if (rc != MRL_OK) return rc;
  TopArgs a = {logits, row_stride, target_ids, token_mask, N, V, k, s.split, s.slice, (float)(1.4426950408889634 / (double)temperature),
               out_ids, out_top_logp, out_logp, out_lse, out_entropy, nullptr, nullptr};
  if (s.split > 1) {
    a.parts = static_cast<Part*>(workspace);
    a.keys = reinterpret_cast<uint64_t*>(static_cast<unsigned char*>(workspace) + parts_bytes(N, s.split));
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  auto go = [&](auto kernel, int threads, int64_t groups) { hipLaunchKernelGGL(kernel, grid_of(groups), dim3(threads), 0, st, a); };
  const bool bf16 = dtype == MRL_BF16;
  if (short_rows(s.split, V, k)) go(bf16 ? k_top<true, kFewThreads> : k_top<false, kFewThreads>, kFewThreads, N);
  else go(bf16 ? k_top<true, kMostThreads> : k_top<false, kMostThreads>, kMostThreads, N * s.split);
  if (s.split > 1) go(bf16 ? k_top_join<true> : k_top_join<false>, kMostThreads, N);
  return hipGetLastError() == hipSuccess ? MRL_OK : MRL_ERR_DEVICE;
}
