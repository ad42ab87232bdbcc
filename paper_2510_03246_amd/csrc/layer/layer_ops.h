// Shared by the forward operators of a decoder layer (linear, layer norm, attention, token log probabilities).
#pragma once

#include "../strp_internal.h"

namespace strp {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef unsigned int uintx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// The stream of a context may be the null stream, which is that of the current device: an operator makes its context's
// device current while it enqueues and leaves the caller's as it was.
class OnDevice {
  int was_ = -1;
  bool ok_ = false;

 public:
  explicit OnDevice(const strp_ctx* ctx) {
    int now = -1;
    if (hipGetDevice(&now) != hipSuccess) return;
    if (now != ctx->device) {
      if (hipSetDevice(ctx->device) != hipSuccess) return;
      was_ = now;
    }
    ok_ = true;
  }
  ~OnDevice() {
    if (was_ >= 0) (void)hipSetDevice(was_);
  }
  bool ok() const { return ok_; }
  OnDevice(const OnDevice&) = delete;
  OnDevice& operator=(const OnDevice&) = delete;
};

static inline bool known_dtype(int dt) { return dt == STRP_BF16 || dt == STRP_F32; }
// A launch has fewer than 2^32 threads: blocks of up to 512 that are surely within it.
constexpr long long MAX_TILES = (1LL << 23) - 1;
static inline size_t bytes_of(int dt) { return dt == STRP_BF16 ? 2 : 4; }
static inline bool ptr16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
static inline bool token_ld(int64_t ld, int64_t T) { return ld >= T && ld % 8 == 0; }

// N consecutive values as floats; N * sizeof(T) bytes aligned to themselves or to 16
template <int N, typename T>
__device__ __forceinline__ void load_floats(const T* p, float (&v)[N]) {
  typedef T vec __attribute__((ext_vector_type(N)));
  const vec x = *(const vec*)p;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (float)x[i];
}
// values rounded once, to the nearest
template <int N, typename T>
__device__ __forceinline__ void store_floats(T* p, const float (&v)[N]) {
  typedef T vec __attribute__((ext_vector_type(N)));
  vec x;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = (T)v[i];
  *(vec*)p = x;
}

// ---- operands of bf16 on their way to the matrix cores ----
typedef short short4v __attribute__((ext_vector_type(4)));

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// 16 bytes per lane from memory to LDS at lds_addr + 16 lane, without registers; completion by wait_loads
__device__ __forceinline__ void copy_to_lds(const void* gptr, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds_addr), "v"(gptr) : "memory", "m0");
}
// the same from a uniform address and a lane's offset in bytes
__device__ __forceinline__ void copy_to_lds_from(const void* base, unsigned lane_off, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds_addr), "v"(lane_off), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop
// all but the last N loads have arrived
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads_and_lds() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(N) : "memory");
}
// lane i of each group of 16 gets column i of the four rows whose 32 bytes the group's lanes 0-3, 4-7, 8-11, 12-15 point at (8 bytes each)
__device__ __forceinline__ short4v read_turned(unsigned lds_addr) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(size_t)lds_addr);
}

}  // namespace strp
