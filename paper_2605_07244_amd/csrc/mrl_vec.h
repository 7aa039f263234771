// Elements of float and bfloat16 tensors eight (or four) at a time, and sums and maxima over lanes: what the row and
// update kernels share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mrl {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Vector accesses at the alignment of one element: rows of odd widths and slices of flat buffers begin anywhere.  gfx950
// takes global accesses of 8 and 16 bytes at any address, so an aligned tensor loses nothing by it.
template <class V, int kAlign> struct __attribute__((packed, aligned(kAlign))) AtAnyAddress { V v; };
template <int kAlign, class V> __device__ inline V load_any(const void* p) { return static_cast<const AtAnyAddress<V, kAlign>*>(p)->v; }
template <int kAlign, class V> __device__ inline void store_any(void* p, V v) { static_cast<AtAnyAddress<V, kAlign>*>(p)->v = v; }
// The same for what nothing near will read again.
template <int kAlign, class V> __device__ inline V load_stream(const void* p) {
  typedef V Unaligned __attribute__((aligned(kAlign)));
  return __builtin_nontemporal_load(static_cast<const Unaligned*>(p));
}
template <int kAlign, class V> __device__ inline void store_stream(void* p, V v) {
  typedef V Unaligned __attribute__((aligned(kAlign)));
  __builtin_nontemporal_store(v, static_cast<Unaligned*>(p));
}

__device__ inline float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ inline uint32_t pack_bf16(float lo, float hi) {          // nearest even; NaN stays NaN
  const __bf16 a = (__bf16)lo, b = (__bf16)hi;
  return (uint32_t)__builtin_bit_cast(uint16_t, a) | (uint32_t)__builtin_bit_cast(uint16_t, b) << 16;
}
// Four e4m3 codes (OCP: no infinities, largest 448), nearest even, of values up to 448.
__device__ inline uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// The eight columns of a row of d that a thread looks at.  Its own are c .. c + 7 as far as the row reaches; at the row's end it looks at the last
// eight of it, of which the first `skip` are other threads' (all eight where c is behind the row).  So every load is whole, inside the row and behind
// no branch: a branch that some lanes take waits for the loads in flight (166666 rows of 384 by 64 lanes, a quarter of them idle: a backward
// pass of 215 us with such branches, 107 without).  Rows of fewer than eight columns are loaded one by one.
struct Columns {
  int at, skip;
  __device__ Columns(int c, int d) : at(max(min(c, d - 8), 0)), skip(c - at) {}
  __device__ bool own(int e, int d) const { return e >= skip && at + e < d; }
};

// Those columns as they lie in memory.
template <bool kBf16> struct Eight;
template <> struct Eight<true> {
  u32x4 w;
  __device__ void load(const void* row, const Columns& c) { w = load_any<2, u32x4>(static_cast<const uint16_t*>(row) + c.at); }
  __device__ void load_short(const void* row, int d) {
    const uint16_t* p = static_cast<const uint16_t*>(row);
    w = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < d) w[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
  }
  __device__ float operator[](int e) const { return e & 1 ? bf16_high(w[e >> 1]) : bf16_low(w[e >> 1]); }
};
template <> struct Eight<false> {
  u32x4 w[2];
  __device__ void load(const void* row, const Columns& c) {
    const float* p = static_cast<const float*>(row) + c.at;
    w[0] = load_any<4, u32x4>(p);
    w[1] = load_any<4, u32x4>(p + 4);
  }
  __device__ void load_short(const void* row, int d) {
    const uint32_t* p = static_cast<const uint32_t*>(row);
    w[0] = w[1] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < d) w[e >> 2][e & 3] = p[e];
  }
  __device__ float operator[](int e) const { return __uint_as_float(w[e >> 2][e & 3]); }
};

template <bool kStream, int kAlign, class V> __device__ inline void store_as(void* p, V v) {
  if (kStream) store_stream<kAlign>(p, v); else store_any<kAlign>(p, v);
}
// The thread's own ones of those columns, of a row of d.  The end of a row, the last n = 8 - skip of the eight, goes out as four, two and one of
// them, as n has bits: what is left below the four or the two begins at an odd element, if it is one.
template <bool kStream = false> __device__ inline void store_eight(void* row, bool bf16, const Columns& c, int d, const float (&v)[8]) {
  const int n = 8 - c.skip;
  const bool four = n & 4;
  if (bf16) {
    uint16_t* p = static_cast<uint16_t*>(row) + c.at;
    const u32x4 w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    if (c.skip == 0 && d >= 8) {
      store_as<kStream, 2>(p, w);
    } else if (d < 8) {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (c.own(e, d)) p[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
    } else if (n > 0) {
      if (four) store_any<2>(p + 4, u32x2{w[2], w[3]});
      if (n & 2) store_any<2>(p + (four ? 2 : 6), four ? w[1] : w[3]);
      if (n & 1) p[c.skip] = (uint16_t)((c.skip < 4 ? c.skip < 2 ? w[0] : w[1] : c.skip < 6 ? w[2] : w[3]) >> 16);
    }
  } else {
    float* p = static_cast<float*>(row) + c.at;
    const u32x4 lo = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    const u32x4 hi = {__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
    if (c.skip == 0 && d >= 8) {
      store_as<kStream, 4>(p, lo);
      store_as<kStream, 4>(p + 4, hi);
    } else if (d < 8) {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (c.own(e, d)) p[e] = v[e];
    } else if (n > 0) {
      if (four) store_any<4>(p + 4, hi);
      if (n & 2) store_any<4>(p + (four ? 2 : 6), four ? u32x2{lo[2], lo[3]} : u32x2{hi[2], hi[3]});
      if (n & 1) store_any<4>(p + c.skip, c.skip < 4 ? c.skip < 2 ? lo[1] : lo[3] : c.skip < 6 ? hi[1] : hi[3]);
    }
  }
}
__device__ inline void store_eight_e4m3(void* row, const Columns& c, int d, const float (&v)[8]) {
  uint8_t* p = static_cast<uint8_t*>(row) + c.at;
  const u32x2 w = {pack_e4m3(v[0], v[1], v[2], v[3]), pack_e4m3(v[4], v[5], v[6], v[7])};
  const int n = 8 - c.skip;
  const bool four = n & 4;
  if (c.skip == 0 && d >= 8) {
    store_any<1>(p, w);
  } else if (d < 8) {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (c.own(e, d)) p[e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
  } else if (n > 0) {
    if (four) store_any<1>(p + 4, w[1]);
    if (n & 2) store_any<1>(p + (four ? 2 : 6), (uint16_t)((four ? w[0] : w[1]) >> 16));
    if (n & 1) p[c.skip] = (uint8_t)((c.skip < 4 ? w[0] : w[1]) >> (8 * (c.skip & 3)));
  }
}

// Over neighbouring lanes, 8, 16, 32 or all 64 of a wave.  Lanes that a step pairs add the same two numbers, so all lanes end with the same bits.
template <int kControl> __device__ inline uint32_t moved(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kControl, 0xf, 0xf, true);
}
constexpr int kSwapOne = 0xB1, kSwapTwo = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;      // quads permuted; 8 and 16 lanes reversed
template <int kLanes, class T, class F> __device__ inline T over_lanes(T x, F join) {
  auto with = [&](uint32_t other) { x = join(x, __builtin_bit_cast(T, other)); };
  with(moved<kSwapOne>(__builtin_bit_cast(uint32_t, x)));
  with(moved<kSwapTwo>(__builtin_bit_cast(uint32_t, x)));
  with(moved<kHalfMirror>(__builtin_bit_cast(uint32_t, x)));
  if (kLanes >= 16) with(moved<kMirror>(__builtin_bit_cast(uint32_t, x)));
  if (kLanes == 32) with(__shfl_xor(__builtin_bit_cast(uint32_t, x), 16));
  if (kLanes == 64) {
    T part[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) part[k] = __builtin_bit_cast(T, (uint32_t)__builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 16 * k));
    x = join(join(part[0], part[1]), join(part[2], part[3]));
  }
  return x;
}
template <int kLanes> __device__ inline float lanes_sum(float x) {
  return over_lanes<kLanes>(x, [](float a, float b) { return a + b; });
}
// Maxima of absolute values as their bits, whose order is that of the values, with infinity above all numbers and NaN above
// infinity: a NaN is kept, where a maximum of floats would drop it.
__device__ inline uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ inline uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }
template <int kLanes> __device__ inline uint32_t lanes_max(uint32_t x) { return over_lanes<kLanes>(x, larger); }

// Scales of e4m3 values: the largest magnitude, at least 2^-100 (whose inverse times 448 still is a number), maps to 448.
constexpr float kE4m3Max = 448.f;
constexpr uint32_t kScaleLeast = (127u - 100u) << 23;

}  // namespace mrl
