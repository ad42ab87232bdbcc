// Shared by the two ways in which attention over a paged cache takes its rows: 16 at a time (cache_rows.hip) and 128 at a time (cache_wide.h).
#pragma once

#include "paged_cache.h"

namespace strp {

constexpr int ROWS = 16, WIDE = 128;
constexpr int WIDE_FROM = 32;              // rows that share keys
constexpr int WORKERS = 512;               // two workgroups a CU
constexpr float LOG2E = 1.44269504088896341f;

struct RowsP {
  Pages c;
  const void* Q;
  void* C;
  const void* K;
  const void* V;
  const floatx4* sK;       // (lowest, step) of two keys
  const floatx4* sV;
  const int32_t* kv_of_head;
  int heads, group;
  long long ldq, ldc;
  float scale_log2e;
  int least, wide_least;   // the fewest units that a workgroup gets
  int wide;                // more than WIDE_FROM rows that share keys are taken 128 at a time, by workgroups of their own
  // what workgroups leave unfinished: [WORKERS][2], of a tile of rows that began before (0) or goes on behind (1)
  float* part;             // [slot][row][channels]
  float2* ml;              // [slot][row]
  long long* off;          // [slot][row] where the row's results go, -1: no such row
  int* parts;              // [worker] how many workgroups share the tile that begins in slot 1; 0: none
  // the same of the tiles of 128
  float* wide_part;        // [slot][channel][row]
  float2* wide_ml;
  long long* wide_off;
  int* wide_parts;
};

// The heads that read a key-value head: `order` has the heads by it, `first` where each one's begin (both null: equal groups).
struct Heads {
  const unsigned short* order;
  const int* first;
  int group;
  __device__ __forceinline__ int of(int kv) const { return first ? first[kv + 1] - first[kv] : group; }
  __device__ __forceinline__ int head(int kv, int i) const { return first ? order[first[kv] + i] : kv * group + i; }
};

__device__ __forceinline__ float both_16(float x, bool sum) {      // with the lane 16 further in its half
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  const unsigned a = r[0], b = r[1];
  return sum ? __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b) : __builtin_elementwise_maximum(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
__device__ __forceinline__ float both_32(float x, bool sum) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  const unsigned a = r[0], b = r[1];
  return sum ? __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b) : __builtin_elementwise_maximum(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
// over the four lanes that have the same row
__device__ __forceinline__ float quads_max(float x) { return both_32(both_16(x, false), false); }
__device__ __forceinline__ float quads_sum(float x) { return both_32(both_16(x, true), true); }

// Exponents in bf16 are S scale - R with R = m scale, rounded: one instruction from a score S and the row's maximum m.  What that rounding took, m scale - R, is in every exponent by m, so results by
// different maxima are brought together with it (else a part's weight is off by up to 2^-24 of its score in powers of two, and from scores of 10^9 on beyond what exp2 holds).
// From R of FAR on differences come first: S is given less m, and R is 0.  In fp32 they always do.
constexpr float FAR = 1048576.0f;          // 2^20: what is left is 2^-5 at most
template <bool BF>
__device__ __forceinline__ float left_over(float m, float scale) {
  const float r = m * scale;
  return BF && fabsf(r) < FAR ? __builtin_fmaf(m, scale, -r) : 0.0f;
}
// what results by the maximum m are multiplied by to be such by `to`, which is not below it: as exponents by that are rounded, or, for those who join them, as if they were not
template <bool BF>
__device__ __forceinline__ float between(float m, float to, float scale) {
  return __builtin_amdgcn_exp2f((m - to) * scale + (left_over<BF>(to, scale) - left_over<BF>(m, scale)));
}
template <bool BF>
__device__ __forceinline__ float between_exactly(float m, float to, float scale) {
  return __builtin_amdgcn_exp2f((m - to) * scale - left_over<BF>(m, scale));
}

// a value that all lanes have, in scalar registers
__device__ __forceinline__ long long uniform(long long x) {
  const unsigned lo = __builtin_amdgcn_readfirstlane((int)x), hi = __builtin_amdgcn_readfirstlane((int)(x >> 32));
  return (long long)((unsigned long long)hi << 32 | lo);
}

// Memory of the device as such: a pointer of which the compiler does not know that is read by loads that count as those of LDS too, and everything is waited for at once.
template <typename T>
using Global = const __attribute__((address_space(1))) T*;
// a base that stays in scalar registers beside its lanes' offsets (or the sums of both that do not change are kept in vector registers, two for an address)
__device__ __forceinline__ Global<char> opaque(const void* p) {
  Global<char> g = (Global<char>)uniform((long long)p);
  asm("" : "+s"(g));
  return g;
}

__device__ __forceinline__ unsigned pick(unsigned a, unsigned b, unsigned sel) { return __builtin_amdgcn_perm(b, a, sel); }
constexpr unsigned LOWS = 0x05040100u, HIGHS = 0x07060302u;      // the lower, the upper halves of a and b
// Whole numbers 0..15 in bits 3-6 and 19-22 as bf16 of 16 + n, which is exact: one instruction where one of the constants is in a vector register, two where both are known.  What 16 times the
// weights adds is taken off behind the sums, of which it is two thirds on average (128 + n, from bits 0-3, would spare a shift in four and make the sums' roundings ten times as large).
struct Numbers16 {
  unsigned of_16 = 0x41804180u;
  __device__ __forceinline__ Numbers16() { asm("" : "+v"(of_16)); }
  __device__ __forceinline__ unsigned operator()(unsigned x) const { return (x & 0x00780078u) | of_16; }
  // the number at `nibble` of either half
  __device__ __forceinline__ unsigned operator()(unsigned x, int nibble) const { return (*this)(nibble ? x >> (4 * nibble - 3) : x << 3); }
};

}  // namespace strp
