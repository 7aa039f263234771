// Embedding lookup with a scale, and its gradient by sorted tokens.
//   y[n, :] = scale * table[id_n, :]            d_table[v, :] (+)= scale * sum over n with id_n = v of dy[n, :]
// Both are bound by memory.  The gradient reads dy once, in the order of the tokens' ids: a stable radix sort of (id, n) by nine bits at a time
// (two passes up to V = 262143, three above; up to kItems tokens in one workgroup and one launch), then waves that each add the rows of a chunk of the
// sorted tokens, 512 columns wide.  A token whose rows lie in one chunk is written from there; of one that reaches over several each chunk
// leaves a partial sum, and a last launch adds them in their order: every sum has a fixed order, no floating-point atomics.
#include "../../include/mrl.h"
#include "mrl_internal.h"
#include "mrl_vec.h"

namespace mrl {
namespace {

constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kRounds = 4;
constexpr int kItems = kSortThreads * kRounds;           // tokens of a workgroup of the sort
constexpr int kWaveItems = 64 * kRounds;
constexpr int64_t kMostTokens = 1 << 24;                  // of a backward call
constexpr int kTileColumns = 512;

// ----------------------------------------------------------------------------
// Lookup: eight columns per thread and vector, kPerThread vectors each.  Four of them where they leave as 16 bytes each, one where they leave as 32
// (32768 tokens, V = 151936, us, four, two and one: 3584 columns bf16 73, 78 and 90; 4096 floats 173, 163 and 149, 713 floats 26.5, 25.4 and 25.0).
// ----------------------------------------------------------------------------
constexpr int kLookThreads = 256;
struct LookArgs {
  const void* table; const int32_t* ids; const uint8_t* mask; int64_t N; int d, V, vectors; float scale; int y_bf16; void* y;
};
template <bool kBf16, int kPerThread> __global__ __launch_bounds__(kLookThreads) void k_embedding(LookArgs a) {
  const int64_t first = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kLookThreads * kPerThread);
  const int64_t n0 = first / a.vectors;                   // (the same for all threads; from there on 32 bits do)
  const int off = (int)(first - n0 * a.vectors);
  Eight<kBf16> x[kPerThread];
  int64_t row[kPerThread];
  int col[kPerThread];
  bool there[kPerThread];
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    const int q = off + j * kLookThreads + (int)threadIdx.x;
    row[j] = n0 + q / a.vectors;
    col[j] = q % a.vectors * 8;
    const int64_t n = row[j] < a.N ? row[j] : a.N - 1;
    const int id = a.ids[n];
    there[j] = id >= 0 && id < a.V && (a.mask == nullptr || a.mask[n] != 0);
    const char* from = static_cast<const char*>(a.table) + (int64_t)(there[j] ? id : 0) * a.d * (kBf16 ? 2 : 4);
    if (a.d >= 8) x[j].load(from, Columns(col[j], a.d)); else x[j].load_short(from, a.d);
  }
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    if (row[j] >= a.N) continue;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = there[j] ? a.scale * x[j][e] : 0.f;
    store_eight(static_cast<char*>(a.y) + row[j] * a.d * (a.y_bf16 ? 2 : 4), a.y_bf16, Columns(col[j], a.d), a.d, v);
  }
}

// ----------------------------------------------------------------------------
// The sort.  Tokens that do not count (masked, or with an id outside [0, V)) have the key V and end up behind the others.
// ----------------------------------------------------------------------------
struct SortArgs {
  const int32_t* ids; const uint8_t* mask; int64_t N; int V, blocks, passes;
  int32_t *key_a, *at_a, *key_b, *at_b;                   // [N] each
  uint32_t* counts;                                       // [blocks][kDigits], of the pass under way
  uint8_t* used;                                          // [V]: 1 where a token occurs (nullptr: not wanted)
};
__device__ inline int key_of(const SortArgs& a, int64_t n) {
  const int id = a.ids[n];
  return id >= 0 && id < a.V && (a.mask == nullptr || a.mask[n] != 0) ? id : a.V;
}

// (the marks are padded to whole vectors)
__device__ inline void clear_marks(const SortArgs& a, int64_t first, int64_t step) {
  for (int64_t v = first; v * 16 < a.V; v += step) reinterpret_cast<u32x4*>(a.used)[v] = u32x4{0, 0, 0, 0};
}

struct SortShared {
  uint16_t table[kSortWaves][kDigits];                    // per wave and digit: a count, then the number of those in earlier waves
  uint32_t start[kDigits];                                // where the block's first item of a digit goes
  uint32_t sums[kSortWaves];
};
// The items' places among those of their digit and wave, the table of earlier waves, and per digit (threads below kDigits) the block's count.
// Item r of a thread is the block's (wave * kWaveItems + 64 r + lane)-th.
__device__ inline uint32_t rank_items(SortShared& sh, const int (&digit)[kRounds], const bool (&valid)[kRounds], int (&place)[kRounds]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  volatile uint16_t* const mine = sh.table[wave];
  for (int i = lane; i < kDigits; i += 64) mine[i] = 0;
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    unsigned long long same = __ballot(valid[r]);
    if (same == 0) continue;
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
      const bool bit = (digit[r] >> b) & 1;
      const unsigned long long set = __ballot(bit);
      same &= bit ? set : ~set;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int before = __popcll(same & ((1ull << lane) - 1ull)), old = mine[digit[r]];
    place[r] = old + before;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (valid[r] && before == 0) mine[digit[r]] = (uint16_t)(old + __popcll(same));
  }
  __syncthreads();
  uint32_t total = 0;
  if (threadIdx.x < kDigits) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = sh.table[w][threadIdx.x];
      sh.table[w][threadIdx.x] = (uint16_t)total;         // (below kItems)
      total += c;
    }
  }
  return total;
}
// Exclusive sums over the digits' numbers (of threads below kDigits); all threads call it.  Holds two barriers.
__device__ inline uint32_t before_digit(SortShared& sh, uint32_t x) {
  uint32_t incl = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t up = __shfl_up(incl, off);
    if ((int)(threadIdx.x & 63) >= off) incl += up;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 63) sh.sums[threadIdx.x >> 6] = incl;
  __syncthreads();
  const uint32_t wave_sum = sh.sums[threadIdx.x & (kSortWaves - 1)];
#pragma unroll
  for (int w = 0; w < kDigits / 64; ++w) incl += w < (int)(threadIdx.x >> 6) ? __builtin_amdgcn_readlane(wave_sum, w) : 0;
  return incl - x;
}

// Counts of a pass's digits, a workgroup per kItems items; with the first the marks are cleared.  (Counts of the second pass made by the first one's stores, with
// atomics in memory, took 25 us of 65536 tokens, for the most common token's 3800 that meet in one; a launch more takes 5.)
__global__ __launch_bounds__(kSortThreads) void k_sort_count(SortArgs a, int pass) {
  __shared__ uint32_t count[kDigits];
  if (threadIdx.x < kDigits) count[threadIdx.x] = 0;
  __syncthreads();
  const int32_t* const from = pass & 1 ? a.key_a : a.key_b;
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t n = (int64_t)blockIdx.x * kItems + r * kSortThreads + threadIdx.x;
    if (n < a.N) atomicAdd(&count[((pass == 0 ? key_of(a, n) : from[n]) >> (pass * kDigitBits)) & (kDigits - 1)], 1u);
  }
  __syncthreads();
  if (threadIdx.x < kDigits) a.counts[(int64_t)blockIdx.x * kDigits + threadIdx.x] = count[threadIdx.x];
  if (pass == 0 && a.used != nullptr) clear_marks(a, (int64_t)blockIdx.x * kSortThreads + threadIdx.x, (int64_t)gridDim.x * kSortThreads);
}

// A pass: every item to its place by the pass's digit, equal ones in their order.  The first reads the tokens and marks them.  Every workgroup adds up the counts of all, which saves a
// launch and grows with the square of N (V = 151936, d = 8 in bf16, us: 2^18 tokens 82, 2^20 172, 2^22 696, 2^24 4830).
__global__ __launch_bounds__(kSortThreads) void k_sort_pass(SortArgs a, int pass) {
  __shared__ SortShared sh;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, shift = pass * kDigitBits;
  const int32_t *const from_key = pass & 1 ? a.key_a : a.key_b, *const from_at = pass & 1 ? a.at_a : a.at_b;
  int32_t *const to_key = pass & 1 ? a.key_b : a.key_a, *const to_at = pass & 1 ? a.at_b : a.at_a;
  int key[kRounds], at[kRounds], digit[kRounds], place[kRounds];
  bool valid[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t n = (int64_t)blockIdx.x * kItems + wave * kWaveItems + r * 64 + lane;
    valid[r] = n < a.N;
    const int64_t m = valid[r] ? n : 0;
    key[r] = pass == 0 ? key_of(a, m) : from_key[m];
    at[r] = pass == 0 ? (int)m : from_at[m];
    digit[r] = (key[r] >> shift) & (kDigits - 1);
    if (pass == 0 && a.used != nullptr && valid[r] && key[r] < a.V) a.used[key[r]] = 1;
  }
  rank_items(sh, digit, valid, place);
  // items of smaller digits, and of this one in earlier blocks
  uint32_t all = 0, earlier = 0;
  if (threadIdx.x < kDigits) {
    const uint32_t* c = a.counts + threadIdx.x;
#pragma unroll 8
    for (int b = 0; b < a.blocks; ++b) {
      const uint32_t x = c[(int64_t)b * kDigits];
      earlier += b < (int)blockIdx.x ? x : 0;
      all += x;
    }
  }
  const uint32_t smaller = before_digit(sh, all);
  if (threadIdx.x < kDigits) sh.start[threadIdx.x] = smaller + earlier;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    if (!valid[r]) continue;
    const uint32_t to = sh.start[digit[r]] + sh.table[wave][digit[r]] + (uint32_t)place[r];
    to_key[to] = key[r];
    to_at[to] = at[r];
  }
}

// 16 bytes of zeros, as far as they lie before `bytes` (a multiple of 2).
__device__ inline void zero_16(char* p, int64_t o, int64_t bytes) {
  if (o + 16 <= bytes) {
    store_any<2>(p + o, u32x4{0, 0, 0, 0});
  } else {
    for (; o < bytes; o += 2) *reinterpret_cast<uint16_t*>(p + o) = 0;
  }
}
// Zeros go out as one store per thread and as many workgroups as that makes: 2.5 GB, us, one and four stores per thread of 256: 367 and 418, of 1024: 395 and 443.
constexpr int64_t kFillBytes = 16 * kSortThreads;

// All of it for at most kItems tokens, by the first workgroup; the result in key_a, at_a.  The others clear the table meanwhile, all of it: the few rows that tokens
// occur in are written twice, which costs less than the sort does (3001 tokens, 32000 x 713 floats: 47 us with marks of the rows and their zeros behind the sort, 30).
__global__ __launch_bounds__(kSortThreads) void k_sort_few(SortArgs a, void* out, int64_t out_bytes) {
  __shared__ SortShared sh;
  __shared__ int32_t keys[kItems], ats[kItems];
  const int64_t group = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (group > 0) { zero_16(static_cast<char*>(out), (group - 1) * kFillBytes + threadIdx.x * 16, out_bytes); return; }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int key[kRounds], at[kRounds], digit[kRounds], place[kRounds];
  bool valid[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int n = wave * kWaveItems + r * 64 + lane;
    valid[r] = n < a.N;
    at[r] = n;
    key[r] = valid[r] ? key_of(a, n) : a.V;               // (no tokens at all: no ids either)
  }
  for (int pass = 0; pass < a.passes; ++pass) {
    const int shift = pass * kDigitBits;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) digit[r] = (key[r] >> shift) & (kDigits - 1);
    const uint32_t count = rank_items(sh, digit, valid, place);
    const uint32_t smaller = before_digit(sh, count);
    if (threadIdx.x < kDigits) sh.start[threadIdx.x] = smaller;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      if (!valid[r]) continue;
      const uint32_t to = sh.start[digit[r]] + sh.table[wave][digit[r]] + (uint32_t)place[r];
      keys[to] = key[r];
      ats[to] = at[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const int n = wave * kWaveItems + r * 64 + lane;
      if (valid[r]) { key[r] = keys[n]; at[r] = ats[n]; }
    }
    __syncthreads();
  }
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int n = wave * kWaveItems + r * 64 + lane;
    if (valid[r]) { a.key_a[n] = key[r]; a.at_a[n] = at[r]; }
  }
}

// ----------------------------------------------------------------------------
// The sums: a wave adds the rows of a chunk's tokens in 512 columns, eight rows on their way; the workgroups behind clear the rows of tokens that do not occur, at the
// same time.  65536 tokens of 4096 columns in bf16, a table of 151936 floats rows: 550 us for 0.54 GB read and 2.49 GB written, 5.5 TB/s, where a fill reaches 6.9
// and a copy 4.9.  (Streaming stores: 1160.  Four or sixteen rows on their way, or chunks of 32: the same.)
// ----------------------------------------------------------------------------
struct SumArgs {
  const void* dy; const int32_t* key; const int32_t* at; const uint8_t* used;
  int64_t N, chunks; int d, V, chunk /*tokens*/, tiles /*of columns*/; float scale; int accumulate, out_bf16; void* out;
  float* parts;                                           // [chunks][2][tiles * kTileColumns]: sums of the first token's rows if it comes from the chunk before,
  int64_t sum_blocks;                                     // and of the last one's if it begins here and goes on
  int wave_rows;                                          // zeros: a wave per row
};
constexpr int kWaveRow = 1024;                            // bytes of a row that a wave clears

__device__ inline void put(const SumArgs& a, int id, const Columns& c, const float (&acc)[8]) {
  char* row = static_cast<char*>(a.out) + (int64_t)id * a.d * (a.out_bf16 ? 2 : 4);
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = a.scale * acc[e];
  if (a.accumulate) {
    Eight<false> old;
    if (a.d >= 8) old.load(row, c); else old.load_short(row, a.d);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += old[e];
  }
  store_eight(row, a.out_bf16, c, a.d, v);
}

template <bool kBf16> __global__ __launch_bounds__(256) void k_embedding_sum(SumArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (block >= a.sum_blocks) {
    // rows of tokens that do not occur, a workgroup each, or a short one a wave
    const int row_bytes = a.d * (a.out_bf16 ? 2 : 4), lanes = a.wave_rows ? 64 : 256;
    const int64_t item = block - a.sum_blocks, v = a.wave_rows ? item * 4 + (threadIdx.x >> 6) : item;
    if (v >= a.V || a.used[v] != 0) return;
    for (int o = (int)(threadIdx.x & (lanes - 1)) * 16; o < row_bytes; o += lanes * 16) zero_16(static_cast<char*>(a.out) + v * row_bytes, o, row_bytes);
    return;
  }
  const int64_t task = block * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = task / a.tiles;
  if (c >= a.chunks) return;
  const int tile = (int)(task - c * a.tiles), col = tile * kTileColumns + lane * 8;
  const int64_t first = c * a.chunk;
  const int n = (int)(a.N - first < a.chunk ? a.N - first : a.chunk);
  const int key = lane < n ? a.key[first + lane] : a.V, at = lane < n ? a.at[first + lane] : 0;
  const int prev = first > 0 ? a.key[first - 1] : -1, next = first + n < a.N ? a.key[first + n] : a.V;
  const int valid = __popcll(__ballot(key < a.V));        // (sorted: the first of them)
  if (valid == 0) return;
  const Columns cols(col, a.d);
  const bool live = col < a.d;
  constexpr int kAhead = 8;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  bool whole = __builtin_amdgcn_readlane(key, 0) != prev; // the run under way began in this chunk
  for (int i0 = 0; i0 < valid; i0 += kAhead) {
    Eight<kBf16> x[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int i = i0 + j < valid ? i0 + j : valid - 1;
      const char* row = static_cast<const char*>(a.dy) + (int64_t)__builtin_amdgcn_readlane(at, i) * a.d * (kBf16 ? 2 : 4);
      if (a.d >= 8) x[j].load(row, cols); else x[j].load_short(row, a.d);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int i = i0 + j;
      if (i >= valid) break;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += x[j][e];
      const int id = __builtin_amdgcn_readlane(key, i);
      const int after = i + 1 < n ? __builtin_amdgcn_readlane(key, i + 1 < 63 ? i + 1 : 63) : next;
      const bool goes_on = i + 1 == n && after == id;
      if (after == id && !goes_on) continue;
      if (whole && !goes_on) {
        if (live) put(a, id, cols, acc);
      } else {
        float* p = a.parts + ((c * 2 + (whole ? 1 : 0)) * a.tiles * kTileColumns) + col;
        *reinterpret_cast<float4*>(p) = make_float4(acc[0], acc[1], acc[2], acc[3]);
        *reinterpret_cast<float4*>(p + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
      }
      whole = true;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    }
  }
}

// Tokens that reach over several chunks: the chunk where one begins adds the partial sums behind its own, four waves a quarter of them each (65536 tokens, the most
// common one in 3800 places: 15 us).
__global__ __launch_bounds__(256) void k_embedding_join(SumArgs a) {
  __shared__ float4 sh[4][2][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t task = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, c = task / a.tiles;
  const int64_t last = (c + 1) * a.chunk;                 // behind the chunk
  if (c >= a.chunks || last >= a.N) return;
  const int id = a.key[last - 1], next = a.key[last], prev = c > 0 ? a.key[c * a.chunk - 1] : -1;
  if (id >= a.V || next != id || prev == id) return;
  const int tile = (int)(task - c * a.tiles), col = tile * kTileColumns + lane * 8;
  const int64_t ld = (int64_t)a.tiles * kTileColumns;
  // the chunks whose first token it is, 64 of them looked up at a time
  int64_t m = 0;
  for (int64_t j0 = c + 1; j0 < a.chunks; j0 += 64) {
    const int64_t j = j0 + lane;
    const unsigned long long same = __ballot(j < a.chunks && a.key[(j < a.chunks ? j : c) * a.chunk] == id);
    m += same == ~0ull ? 64 : __builtin_ctzll(~same);
    if (same != ~0ull) break;
  }
  // part 0 is the chunk's own
  const int64_t per = (m + 1 + 3) / 4, i0 = wave * per, i1 = i0 + per < m + 1 ? i0 + per : m + 1;
  float4 lo = make_float4(0.f, 0.f, 0.f, 0.f), hi = lo;
#pragma unroll 8
  for (int64_t i = i0; i < i1; ++i) {
    const float* q = a.parts + ((c + i) * 2 + (i == 0)) * ld + col;
    const float4 x = *reinterpret_cast<const float4*>(q), y = *reinterpret_cast<const float4*>(q + 4);
    lo.x += x.x; lo.y += x.y; lo.z += x.z; lo.w += x.w;
    hi.x += y.x; hi.y += y.y; hi.z += y.z; hi.w += y.w;
  }
  sh[wave][0][lane] = lo;
  sh[wave][1][lane] = hi;
  __syncthreads();
  if (wave != 0 || col >= a.d) return;
  float acc[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float4 s = sh[0][h][lane];
#pragma unroll
    for (int w = 1; w < 4; ++w) { const float4 x = sh[w][h][lane]; s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w; }
    acc[4 * h] = s.x; acc[4 * h + 1] = s.y; acc[4 * h + 2] = s.z; acc[4 * h + 3] = s.w;
  }
  put(a, id, Columns(col, a.d), acc);
}

// ----------------------------------------------------------------------------
constexpr int64_t kMostRows = (int64_t)1 << 30, kMostWide = 1 << 21;
constexpr int kMostColumns = 1 << 20, kMostIds = 1 << 24;
dim3 grid_of(int64_t groups) {
  const int64_t wide = groups < kMostWide ? groups : kMostWide;
  return dim3((unsigned)wide, (unsigned)((groups + wide - 1) / wide));
}
bool is_float_type(int32_t t) { return t == MRL_F32 || t == MRL_BF16; }

struct BackLayout {
  size_t total = 0, key_a, at_a, key_b, at_b, counts, used, parts;
  int blocks, passes, chunk, tiles;
  int64_t chunks;
};
size_t take(size_t& off, size_t bytes) {
  const size_t at = off;
  off += (bytes + 255) / 256 * 256;
  return at;
}
// Chunks of 64 tokens (a lane each) where they make waves enough for the chip, else of 16, or of 8 where the sort is one launch and the sums' latency counts (us, 16, 8 and 4:
// 3001 tokens, 32000 x 713 floats 28.2, 25.9 and 25.3; into a float table 1000 tokens of 1536 columns 22.5, 18.4 and 17.1, all of them one token 19.3, 19.0 and 24.3; 16000 of 256 45, 45 and 50).
BackLayout layout_of(int64_t N, int d, int V) {
  BackLayout L;
  L.blocks = (int)((N + kItems - 1) / kItems);
  L.passes = V < 1 << kDigitBits ? 1 : V < 1 << 2 * kDigitBits ? 2 : 3;
  L.tiles = (d + kTileColumns - 1) / kTileColumns;
  L.chunk = N <= kItems ? 8 : (N + 63) / 64 * L.tiles >= 2048 ? 64 : 16;
  L.chunks = (N + L.chunk - 1) / L.chunk;
  size_t off = 0;
  L.key_a = take(off, (size_t)N * 4); L.at_a = take(off, (size_t)N * 4);
  L.key_b = take(off, (size_t)N * 4); L.at_b = take(off, (size_t)N * 4);
  L.counts = take(off, (size_t)L.blocks * kDigits * 4);
  L.used = take(off, (size_t)V);
  L.parts = take(off, (size_t)L.chunks * 2 * L.tiles * kTileColumns * 4);
  L.total = off;
  return L;
}
bool back_shape(int64_t N, int32_t d, int32_t V) { return N >= 0 && N <= kMostTokens && d > 0 && d <= kMostColumns && V > 0 && V <= kMostIds; }

}  // namespace
}  // namespace mrl

using namespace mrl;

extern "C" int mrl_embedding(const void* table, const int32_t* ids, const uint8_t* token_mask, int64_t N, int32_t d, int32_t V, float scale,
                             int32_t table_dtype, int32_t y_dtype, void* out_y, void* stream) {
  if (!is_float_type(table_dtype) || !is_float_type(y_dtype)) return MRL_ERR_DTYPE;
  if (N < 0 || N > kMostRows || d <= 0 || d > kMostColumns || V <= 0 || V > kMostIds) return MRL_ERR_SHAPE;
  if (!(scale > -INFINITY && scale < INFINITY)) return MRL_ERR_CONFIG;
  if (N == 0) return MRL_OK;
  if (!table || !ids || !out_y) return MRL_ERR_NULL;
  const int rc = require_gfx950();
  if (rc != MRL_OK) return rc;
  const int vectors = (d + 7) / 8;
  const LookArgs a = {table, ids, token_mask, N, d, V, vectors, scale, y_dtype == MRL_BF16, out_y};
  const int per_group = kLookThreads * (a.y_bf16 ? 4 : 1);
  const dim3 grid = grid_of((N * vectors + per_group - 1) / per_group);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const auto kernel = table_dtype == MRL_BF16 ? (a.y_bf16 ? k_embedding<true, 4> : k_embedding<true, 1>) : a.y_bf16 ? k_embedding<false, 4> : k_embedding<false, 1>;
  hipLaunchKernelGGL(kernel, grid, dim3(kLookThreads), 0, s, a);
  return hipGetLastError() == hipSuccess ? MRL_OK : MRL_ERR_DEVICE;
}

extern "C" size_t mrl_embedding_backward_workspace(int64_t N, int32_t d, int32_t V) {
  if (!back_shape(N, d, V)) return 0;
  return layout_of(N > 0 ? N : 1, d, V).total;
}

extern "C" int mrl_embedding_backward(const void* dy, const int32_t* ids, const uint8_t* token_mask, int64_t N, int32_t d, int32_t V, float scale,
                                      int32_t dy_dtype, int32_t out_dtype, int32_t accumulate, void* out_dtable, void* workspace, size_t workspace_bytes,
                                      void* stream) {
  if (!is_float_type(dy_dtype) || !is_float_type(out_dtype)) return MRL_ERR_DTYPE;
  if (!back_shape(N, d, V)) return MRL_ERR_SHAPE;
  if (!(scale > -INFINITY && scale < INFINITY) || (accumulate != 0 && accumulate != 1) || (accumulate && out_dtype != MRL_F32)) return MRL_ERR_CONFIG;
  if (!out_dtable || (N > 0 && (!dy || !ids))) return MRL_ERR_NULL;
  if (N == 0 && accumulate) return MRL_OK;
  const BackLayout L = layout_of(N > 0 ? N : 1, d, V);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < L.total) return MRL_ERR_WORKSPACE;
  const int rc = require_gfx950();
  if (rc != MRL_OK) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  auto at = [&](size_t off) { return reinterpret_cast<int32_t*>(ws + off); };
  const bool few = N <= kItems;
  uint8_t* const used = accumulate || few ? nullptr : ws + L.used;
  const SortArgs sort = {ids, token_mask, N, V, L.blocks, L.passes, at(L.key_a), at(L.at_a), at(L.key_b), at(L.at_b),
                         reinterpret_cast<uint32_t*>(ws + L.counts), used};
  bool in_a = true;
  if (few) {
    const int64_t bytes = (int64_t)V * d * (out_dtype == MRL_BF16 ? 2 : 4), fill = accumulate ? 0 : (bytes + kFillBytes - 1) / kFillBytes;
    hipLaunchKernelGGL(k_sort_few, grid_of(1 + fill), dim3(kSortThreads), 0, s, sort, out_dtable, bytes);
    if (N == 0) return hipGetLastError() == hipSuccess ? MRL_OK : MRL_ERR_DEVICE;
  } else {
    for (int p = 0; p < L.passes; ++p) {
      hipLaunchKernelGGL(k_sort_count, dim3(L.blocks), dim3(kSortThreads), 0, s, sort, p);
      hipLaunchKernelGGL(k_sort_pass, dim3(L.blocks), dim3(kSortThreads), 0, s, sort, p);
    }
    in_a = L.passes % 2 == 1;
  }
  const int64_t sum_blocks = N > 0 ? (L.chunks * L.tiles + 3) / 4 : 0, row_bytes = (int64_t)d * (out_dtype == MRL_BF16 ? 2 : 4);
  const bool wave_rows = row_bytes <= kWaveRow;
  const int64_t zero_blocks = used == nullptr ? 0 : wave_rows ? ((int64_t)V + 3) / 4 : V;
  const SumArgs a = {dy, in_a ? sort.key_a : sort.key_b, in_a ? sort.at_a : sort.at_b, used, N, L.chunks, d, V, L.chunk, L.tiles, scale, accumulate,
                     out_dtype == MRL_BF16, out_dtable, reinterpret_cast<float*>(ws + L.parts), sum_blocks, wave_rows};
  hipLaunchKernelGGL(dy_dtype == MRL_BF16 ? k_embedding_sum<true> : k_embedding_sum<false>, grid_of(sum_blocks + zero_blocks), dim3(256), 0, s, a);
  if (N > L.chunk) hipLaunchKernelGGL(k_embedding_join, grid_of(L.chunks * L.tiles), dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? MRL_OK : MRL_ERR_DEVICE;
}
