// Shared by the operators on a paged cache of keys and values (append, attention).
#pragma once

#include "layer_ops.h"

namespace strp {

constexpr int MAX_CACHE_HEADS = 1024;

// The cache as kernels see it.  Everything that comes from device memory is brought into its range before it is used.
struct Pages {
  const int32_t* table;
  const int32_t* past;
  const int32_t* seq_start;
  int kv_heads, dh, page_log2, pages, n_seq, ld_table, cap;      // cap: tokens that a sequence's row of the table holds
  int T;
};

__device__ __forceinline__ int clamped(int x, int lo, int hi) { return min(max(x, lo), hi); }
__device__ __forceinline__ int seq_begin(const Pages& c, int s) { return c.seq_start ? clamped(c.seq_start[s], 0, c.T) : (s ? c.T : 0); }
// tokens of the cache before the call's own
__device__ __forceinline__ int seq_past(const Pages& c, int s) { return clamped(c.past[s], 0, c.cap); }

// Errors of the arguments that both operators share; null where there are none.
static inline const char* cache_error(const strp_cache& c, int dtype, int heads, int64_t T) {
  if (!known_dtype(dtype)) return "unknown dtype";
  if (c.format != STRP_CACHE_Q4 && c.format != STRP_CACHE_BF16 && c.format != STRP_CACHE_F32) return "unknown format of the cache";
  if (!c.K || !c.V || !c.table || !c.past) return "null K, V, table or past of the cache";
  if (c.format == STRP_CACHE_Q4 ? !c.K_scale || !c.V_scale : (c.format == STRP_CACHE_BF16) != (dtype == STRP_BF16))
    return c.format == STRP_CACHE_Q4 ? "a cache of 4 bits needs K_scale and V_scale" : "the cache has another type than the activations";
  if (heads <= 0 || c.kv_heads <= 0 || c.d_head <= 0 || T <= 0 || c.pages <= 0 || c.n_seq <= 0 || c.ld_table <= 0) return "sizes must be positive";
  if (c.d_head % 8 || c.d_head > 128) return "d_head must be a multiple of 8 and at most 128";
  if (c.page < 16 || c.page > 65536 || (c.page & (c.page - 1))) return "page must be a power of two from 16 to 65536";
  if ((int64_t)c.ld_table * c.page > (1LL << 30)) return "ld_table * page above 2^30";
  if (heads > MAX_CACHE_HEADS || c.kv_heads > MAX_CACHE_HEADS) return "more than 1024 heads";
  if (c.n_seq > 65536) return "more than 65536 sequences";
  if (T > (1LL << 27)) return "more than 2^27 tokens";
  if (!c.seq_start && c.n_seq != 1) return "no seq_start needs n_seq = 1";
  if (!ptr16(c.K) || !ptr16(c.V) || !ptr16(c.K_scale) || !ptr16(c.V_scale)) return "the cache is not 16-byte aligned";
  return nullptr;
}

static inline Pages pages_of(const strp_cache& c, int64_t T) {
  return Pages{c.table, c.past, c.seq_start, c.kv_heads, c.d_head, __builtin_ctz((unsigned)c.page), c.pages, c.n_seq, c.ld_table, c.ld_table * c.page, (int)T};
}

}  // namespace strp
