// Causal attention over whole prompts, heads in groups, sequences packed along the tokens.
//
//   c_t = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q_t . k_j - m),  j from the start of t's sequence to t,
// in one pass over the keys with the running maximum m and sum of the softmax.  A workgroup has the queries of one head at
// consecutive tokens and walks the keys from the start of its first query's sequence; every query has a range [lo, t] of
// keys, so that a tile of queries that crosses from one sequence into the next needs nothing of its own.
#include "layer_ops.h"

#include <type_traits>

namespace strp {

struct AttnP {
  const void* Q;
  const void* K;
  const void* V;
  void* C;
  const int32_t* seq_start;
  const int32_t* kv_of_head;
  int heads, kv_heads, group, dh, n_seq, tiles;
  long long T, ldq, ldk, ldv, ldc;
  float scale_log2e;
  int near;          // rows of K and V lie near enough for offsets of 32 bits, and come in eights
};

// First key of token t's sequence; t + 1 where t is in none.
__device__ __forceinline__ int first_key(const AttnP& p, int t) {
  if (t >= p.T) return t + 1;
  if (!p.seq_start) return 0;
  int a = -1, b = p.n_seq + 1;             // seq_start[a] <= t < seq_start[b]
  while (b - a > 1) {
    const int c = (a + b) >> 1;
    if (p.seq_start[c] <= t) a = c;
    else b = c;
  }
  if (a < 0 || a == p.n_seq) return t + 1;
  const int s = p.seq_start[a];
  return s < 0 ? 0 : s;
}

__device__ __forceinline__ int kv_head_of(const AttnP& p, int head) {
  if (!p.kv_of_head) return head / p.group;
  const int g = p.kv_of_head[head];
  return g < 0 ? 0 : (g < p.kv_heads ? g : p.kv_heads - 1);
}

// Products of fp32 (v_mfma_f32_32x32x2_f32).  A workgroup has 64 queries, keys 64 at a time: a wavefront has half of either, and the two that have the same
// queries put their maxima, sums and results together at the end.  (128 queries and every wavefront on all the keys: 241 us for 8 heads x 80 over prompts of 1000,
// 513 and 1500 tokens, nearly all of it the row of 24 tiles that the last queries wait for.  32 queries and the four wavefronts on a quarter of the keys each: 190
// us, and 27 TFLOP/s at 128 channels a head, since that is 16 operations for a byte of L2.)  S = K^T Q has a query to a lane (the keys of its 16 registers are
// 8 (e / 4) + 4 (lane / 32) + e % 4), so the softmax needs one exchange between the lane's two halves, and the registers of P are the second operand of V P as
// they are.  What bounds it is the matrix cores, and between tiles the way of K and V to LDS, which a second workgroup on the CU fills: those prompts 156 us, 16 heads of 128 at 93 TFLOP/s.
template <int DHP>
__global__ __launch_bounds__(256, 2) void attention_f32_kernel(const AttnP p) {
  constexpr int KT = 64, PITCH = KT + 4, NC = DHP / 32, CHUNKS = KT / 4;
  __shared__ __attribute__((aligned(16))) float sK[DHP][PITCH], sV[DHP][PITCH];
  __shared__ float sM[2][32], sL[2][32];
  __shared__ int lows[4];
  static_assert(2 * 32 * 33 <= 64 * PITCH, "the other half's results lie where K was");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, l32 = lane & 31;
  const int part = wave >> 1, group = wave & 1;                            // half of the keys, of the queries
  const int slot = (int)blockIdx.x % p.heads, tile = p.tiles - 1 - (int)blockIdx.x / p.heads;       // from the last tile on: of one sequence those with most keys first
  const int head = p.heads % 8 == 0 ? (slot & 7) * (p.heads >> 3) + (slot >> 3) : slot;
  const int q0 = tile * 64, q = q0 + group * 32 + l32, kv = kv_head_of(p, head);
  float qf[DHP / 2];
  {
    const float* Q = (const float*)p.Q + (long long)head * p.dh * p.ldq + (q < p.T ? q : 0);
#pragma unroll
    for (int s = 0; s < DHP / 2; ++s) {
      const int d = 2 * s + h;
      qf[s] = Q[(long long)(d < p.dh ? d : 0) * p.ldq];
    }
  }
  const int lo = first_key(p, q);
#pragma unroll
  for (int s = 0; s < DHP / 2; ++s) {
    qf[s] = 2 * s + h < p.dh ? qf[s] : 0.0f;
    __builtin_amdgcn_sched_barrier(0);                                     // one comparison at a time, or their results take the scalar registers
  }
  int wlo = lo <= q ? lo : 0x7fffffff, whi = wlo;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    wlo = min(wlo, __shfl_xor(wlo, o, 64));
    whi = max(whi, __shfl_xor(whi, o, 64));
  }
  wlo = __builtin_amdgcn_readfirstlane(wlo);
  whi = __builtin_amdgcn_readfirstlane(whi);
  const int wq = q0 + group * 32;
  if (lane == 0) lows[wave] = wlo;
  __syncthreads();
  const int low = min(lows[0], lows[1]);
  if (low == 0x7fffffff) return;                 // no query of this tile is in a sequence
  const int last = q0 + 63 < (int)(p.T - 1) ? q0 + 63 : (int)(p.T - 1);

  floatx16 O[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) O[c][e] = 0.0f;
  float m = -INFINITY, l = 0.0f;
  const float* Kh = (const float*)p.K + (long long)kv * p.dh * p.ldk;
  const float* Vh = (const float*)p.V + (long long)kv * p.dh * p.ldv;
  // the next tile is asked for into registers while this one is worked on, where there are registers for it
  constexpr bool AHEAD = DHP < 128;
  constexpr int ROWS = 256 / CHUNKS, NR = DHP / ROWS;
  const int row0 = tid / CHUNKS, col = (tid % CHUNKS) * 4;
  floatx4 nk[AHEAD ? NR : 4], nv[AHEAD ? NR : 4];
  auto ask = [&](int k0, int first, int n) {
    int r0 = row0;
    asm volatile("" : "+v"(r0));                                           // or every row's address is worked out once and kept
    const float* kp = Kh + (long long)r0 * p.ldk + k0 + col;
    const float* vp = Vh + (long long)r0 * p.ldv + k0 + col;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      nk[i] = nv[i] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
      if (r0 + ROWS * (first + i) < p.dh && k0 + col < p.T) {
        nk[i] = *(const floatx4*)(kp + (long long)(ROWS * (first + i)) * p.ldk);
        nv[i] = *(const floatx4*)(vp + (long long)(ROWS * (first + i)) * p.ldv);
      }
    }
  };
  auto put = [&](int first, int n) {
#pragma unroll
    for (int i = 0; i < n; ++i) {
      *(floatx4*)&sK[row0 + ROWS * (first + i)][col] = nk[i];
      *(floatx4*)&sV[row0 + ROWS * (first + i)][col] = nv[i];
    }
  };
  if constexpr (AHEAD) ask(low & ~(KT - 1), 0, NR);
#pragma unroll 1
  for (int k0 = low & ~(KT - 1); k0 <= last; k0 += KT) {
    __syncthreads();
    if constexpr (AHEAD) {
      put(0, NR);
    } else {
#pragma unroll
      for (int i = 0; i < NR; i += 4) {
        ask(k0, i, 4);
        put(i, 4);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __syncthreads();
    if constexpr (AHEAD)
      if (k0 + KT <= last) ask(k0 + KT, 0, NR);
    const int k1 = k0 + 32 * part;
    if (wq + 31 < k1 || wlo >= k1 + 32) continue;                          // nothing here that this wavefront sees
    const bool whole = whi <= k1 && wq >= k1 + 31;
    floatx16 S;
#pragma unroll
    for (int e = 0; e < 16; ++e) S[e] = 0.0f;
#pragma unroll
    for (int s = 0; s < DHP / 2; ++s) {
      if (s < DHP / 2 - 16 || 2 * s < p.dh) S = __builtin_amdgcn_mfma_f32_32x32x2f32(sK[2 * s + h][32 * part + l32], qf[s], S, 0, 0, 0);
      if (s % 16 == 15) __builtin_amdgcn_sched_barrier(0);       // not every fragment at once, for the registers
    }
    if (!whole)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = k1 + 8 * (e >> 2) + 4 * h + (e & 3);
        if (key < lo || key > q) S[e] = -INFINITY;
      }
    float mt = m;
#pragma unroll
    for (int e = 0; e < 16; ++e) mt = __builtin_elementwise_maximum(mt, S[e]);
    mt = __builtin_elementwise_maximum(mt, __shfl_xor(mt, 32, 64));
    const float fac = mt == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - mt) * p.scale_log2e);
    m = mt;
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      S[e] = __builtin_amdgcn_exp2f((S[e] - (mt == -INFINITY ? 0.0f : mt)) * p.scale_log2e);      // the difference first: it is exact, or small against what it is taken from
      sum += S[e];
    }
    l = l * fac + sum;
    // Where some key is not seen by every query, a value that is not finite would reach those too, by a probability of zero: such values are left out of
    // the products and added to the results of the queries that see them.
    // A tile's share is summed by itself: so the chains that round are as long as a tile and as the number of tiles, not as the keys.
    bool odd = false;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      floatx16 share;
#pragma unroll
      for (int e = 0; e < 16; ++e) share[e] = 0.0f;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        floatx4 v = *(const floatx4*)&sV[32 * c + l32][32 * part + 8 * g + 4 * h];
        if (!whole)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool fin = fabsf(v[e]) < INFINITY;
            odd = odd || !fin;
            v[e] = fin ? v[e] : 0.0f;
          }
#pragma unroll
        for (int e = 0; e < 4; ++e) share = __builtin_amdgcn_mfma_f32_32x32x2f32(v[e], S[4 * g + e], share, 0, 0, 0);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) O[c][e] = __builtin_fmaf(O[c][e], fac, share[e]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (__builtin_amdgcn_ballot_w64(odd))
#pragma unroll 1
      for (int i = 0; i < 32; ++i) {
        const bool seen = k1 + i >= lo && k1 + i <= q;
        if (!__builtin_amdgcn_ballot_w64(seen)) continue;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float v = sV[32 * c + 8 * (e >> 2) + 4 * h + (e & 3)][32 * part + i];
            O[c][e] += seen && !(fabsf(v) < INFINITY) ? v : 0.0f;
          }
      }
  }
  // the second half of the keys to the first: the results 32 channels at a time
  l += __shfl_xor(l, 32, 64);
  __syncthreads();
  if (part == 1 && h == 0) {
    sM[group][l32] = m;
    sL[group][l32] = l;
  }
  float(*other)[32][33] = (float(*)[32][33])&sK[0][0];
  __syncthreads();
  const float m1 = sM[group][l32], l1 = sL[group][l32], most = __builtin_elementwise_maximum(m, m1);
  // a wavefront that saw no key has a sum and results of zero
  const float f0 = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - most) * p.scale_log2e), f1 = m1 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m1 - most) * p.scale_log2e);
  const float inv = 1.0f / (f0 * l + f1 * l1);
  float* C = (float*)p.C + (long long)head * p.dh * p.ldc + q;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    if (part == 1)
#pragma unroll
      for (int e = 0; e < 16; ++e) other[group][8 * (e >> 2) + 4 * h + (e & 3)][l32] = O[c][e];
    __syncthreads();
    if (part == 0 && lo <= q)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int r = 8 * (e >> 2) + 4 * h + (e & 3);
        if (32 * c + r < p.dh) C[(long long)(32 * c + r) * p.ldc] = (f0 * O[c][e] + f1 * other[group][r][l32]) * inv;
      }
    __syncthreads();
  }
}

__device__ const unsigned zero_chunk[4] = {0u, 0u, 0u, 0u};

// Products of bf16 (v_mfma_f32_32x32x16_bf16).  NW wavefronts of 32 queries, keys 64 at a time.  S = K^T Q has a query to a lane.  The fragments of K are read
// turned (K lies with its tokens contiguous), in quads of keys, and which quads a lane's rows are is free: with the middle bits of a quad's number exchanged,
// register e of S is key 16 (e / 8) + 8 (lane / 32) + e % 8, so eight registers of P are a second operand of V P as they are and the fragment of V beside it is
// 16 contiguous bytes.  The chunks of 16 bytes in a row of K or V lie in LDS in an order that depends on the row, so that what is read at once lies in
// different banks.
// What bounds it is the vector unit (an exponential, a multiply-add, an addition, half a maximum and half a conversion for a score) and, at 128 channels a head, as
// much the matrix cores (busy with SPLIT 66 and 36 % of the time at 64 channels, 49 and 50 % at 128; without 57 and 29, 41 and 40).  So that either has work while the other waits, the scores of the next tile are multiplied beside the softmax of this one, and V P follows
// it a quarter of the keys at a time.  K runs a tile ahead of V: LDS has RING tiles of each.
// SPLIT: the probabilities meet V as two terms of bf16, which is half as many matrix instructions again and three vector instructions a score.  With one term results are further from
// those in 64 bits than their own rounding puts them (2.0e-3 against 1.66e-3, relative, on Gaussian V); with two they are not.  Whole calls, two terms / one: eight prompts of 2048 tokens, 32 heads
// of 64: 271 / 221 us; 16221 tokens in prompts of 1 to 8191, 32 heads of 128 on 8: 1101 / 890 us.
template <int DHP, int NW, int RING, int WPS, bool SPLIT>
__global__ __launch_bounds__(64 * NW, WPS) void attention_bf16_kernel(const AttnP p) {
  constexpr int KT = 64, NC = DHP / 32, NS = DHP / 16, TILE = DHP * 128, LH = DHP / 8 / NW, BQ = 32 * NW;      // LH: KBs of a tile of K or V that a wavefront moves
  static_assert(DHP % (8 * NW) == 0, "whole pieces for every wavefront");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * RING * TILE];
  __shared__ int lows[NW];
  constexpr bool QLDS = SPLIT && DHP <= 64;      // Q stays in LDS, for the registers of the second term
  __shared__ bf16x8 sQ[QLDS ? NW : 1][QLDS ? NS : 1][QLDS ? 64 : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, l32 = lane & 31;
  // from the last tile on (of one sequence those with most keys first); the heads that an XCD gets are neighbours where eight divides them, since neighbours share K and V
  const int slot = (int)blockIdx.x % p.heads, tile = p.tiles - 1 - (int)blockIdx.x / p.heads;
  const int head = p.heads % 8 == 0 ? (slot & 7) * (p.heads >> 3) + (slot >> 3) : slot;
  const int q0 = tile * BQ, q = q0 + wave * 32 + l32;
  bf16x8 qf[NS];
  {
    const __bf16* Q = (const __bf16*)p.Q + (long long)head * p.dh * p.ldq + (q < p.T ? q : 0);
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int d = 16 * s + 8 * h + e;
        const __bf16 v = Q[(long long)(d < p.dh ? d : 0) * p.ldq];
        qf[s][e] = d < p.dh ? v : (__bf16)0.0f;
      }
  }
  if constexpr (QLDS)
#pragma unroll
    for (int s = 0; s < NS; ++s) sQ[wave][s][lane] = qf[s];
  const int lo = first_key(p, q);
  // the wavefront's first key, and the first key from which on every query sees (none, if some query is in no sequence)
  int wlo = lo <= q ? lo : 0x7fffffff, whi = wlo;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    wlo = min(wlo, __shfl_xor(wlo, o, 64));
    whi = max(whi, __shfl_xor(whi, o, 64));
  }
  wlo = __builtin_amdgcn_readfirstlane(wlo);
  whi = __builtin_amdgcn_readfirstlane(whi);
  const int wq = q0 + wave * 32;
  if (lane == 0) lows[wave] = wlo;
  __syncthreads();
  int low = lows[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) low = min(low, lows[w]);
  low = __builtin_amdgcn_readfirstlane(low);
  if (low == 0x7fffffff) return;                 // no query of this tile is in a sequence
  const int last = q0 + BQ - 1 < (int)(p.T - 1) ? q0 + BQ - 1 : (int)(p.T - 1);
  const int first = low & ~(KT - 1), steps = (last - first) / KT + 1;

  const int kv = kv_head_of(p, head);
  // a wavefront moves eight rows of K or of V at a time, 8 NW rows apart: lane l has a chunk of row l / 8 of them
  const unsigned base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int row0 = 8 * wave + (lane >> 3);
  const int chunkK = 8 * ((lane & 7) ^ (((row0 >> 1) & 1) << 2)), chunkV = 8 * ((lane & 7) ^ ((row0 >> 1) & 7));
  const __bf16* srcK = (const __bf16*)p.K + (long long)kv * p.dh * p.ldk + first;
  const __bf16* srcV = (const __bf16*)p.V + (long long)kv * p.dh * p.ldv + first;
  // Rows behind the head's and tokens behind the last are zeros; tiles behind the last are not looked at.  A tile that is all there is asked for by
  // lane offsets that stay the same (in 32 bits, if eight rows lie near enough).
  auto issue = [&](const __bf16* src, int chunk, long long ld, int s, unsigned at) {
    const __bf16* from = src + s * KT;
    if (p.near && first + (s + 1) * KT <= (int)p.T) {
      const unsigned off = (unsigned)((row0 * ld + chunk) * 2);
#pragma unroll
      for (int i = 0; i < LH; ++i) {
        const bool rows = 8 * (wave + NW * i) < p.dh;
        copy_to_lds_from(rows ? (const void*)(from + (long long)(8 * NW * i) * ld) : (const void*)zero_chunk, off & (rows ? ~0u : 0u), at + (unsigned)wave * 1024 + NW * 1024 * i);
      }
    } else {
      int r = row0, c = chunk;
      asm volatile("" : "+v"(r), "+v"(c));       // rare: what it works out is not worth registers
      const bool in = first + c + s * KT < (int)p.T;
#pragma unroll
      for (int i = 0; i < LH; ++i) {
        const __bf16* g = from + (r + (long long)(8 * NW * i)) * ld + c;
        copy_to_lds(in && r + 8 * NW * i < p.dh ? (const void*)g : (const void*)zero_chunk, at + (unsigned)wave * 1024 + NW * 1024 * i);
      }
    }
  };
  const unsigned baseV = base + RING * TILE;
  unsigned toK = base, toV = baseV;              // where the next tile goes
  auto issue_k = [&](int s) {
    issue(srcK, chunkK, p.ldk, s, toK);
    toK = toK == base + (RING - 1) * TILE ? base : toK + TILE;
  };
  auto issue_v = [&](int s) {
    issue(srcV, chunkV, p.ldv, s, toV);
    toV = toV == baseV + (RING - 1) * TILE ? baseV : toV + TILE;
  };
  // fragments of K: row 16 s + 8 h + (lane % 16) / 4 (+ 4), quad of keys; of V: row 32 c + lane % 32, chunk 2 k + h
  const int r4 = 4 * ((lane >> 4) & 1) + (lane & 3), key4 = (r4 & 4) | ((r4 & 1) << 1) | ((r4 >> 1) & 1), kr = (lane & 15) >> 2;
  const unsigned offK = (unsigned)((8 * h + kr) * 128 + (kr >> 1) * 64 + (key4 >> 1) * 16 + (key4 & 1) * 8);
  const unsigned offV = (unsigned)(l32 * 128 + ((((l32 >> 1) & 7) ^ h) * 16));
  auto frag_k = [&](unsigned at, int d, int u) {
    const unsigned a = at + (offK ^ (unsigned)(64 * u)) + 2048 * d;
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(read_turned(a), read_turned(a + 512), 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto frag_v = [&](unsigned at, int c, int k) { return *(const __attribute__((address_space(3))) bf16x8*)(size_t)(at + (offV ^ (unsigned)(32 * k)) + 4096 * c); };

  floatx16 O[NC];
  float m, l[2];
  bool again = false;
  struct Scores { floatx16 u[2]; };
  auto clear = [&](Scores& S) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) S.u[u][e] = 0.0f;
  };
  auto sees = [&](int s) { return wq + 31 >= first + s * KT && wlo < first + (s + 1) * KT; };      // some query, perhaps
  auto scores = [&](Scores& S, unsigned at, int d0, int d1) {
#pragma unroll
    for (int d = d0; d < d1; ++d) {
      bf16x8 qd;
      if constexpr (QLDS) qd = sQ[wave][d][lane];
      else qd = qf[d];
#pragma unroll
      for (int u = 0; u < 2; ++u) S.u[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_k(at, d, u), qd, S.u[u], 0, 0, 0);
    }
  };
  // all of them; not every fragment at once, for the registers
  auto all_scores = [&](Scores& S, unsigned at) {
#pragma unroll
    for (int d = 0; d < NS; d += 2) {
      scores(S, at, d, d + 2);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // the running maximum with a tile's scores, what is held rescaled to it; returns what is to be taken from a score in powers of two
  auto raise = [&](const Scores& S) {
    float mt = m;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) mt = __builtin_elementwise_maximum(mt, S.u[u][e]);
    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, mt), __builtin_bit_cast(unsigned, mt), false, false);
    const unsigned b0 = both[0], b1 = both[1];
    mt = __builtin_elementwise_maximum(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
    // What a query holds stays as it is until its maximum has grown past 2^8 times: probabilities of up to 256 are as good as those below 1.
    const bool grown = !((mt - m) * p.scale_log2e <= 8.0f || mt == -INFINITY);
    if (__builtin_amdgcn_ballot_w64(grown)) {
      const float fac = grown ? __builtin_amdgcn_exp2f((m - mt) * p.scale_log2e) : 1.0f;
      l[0] *= fac;
      if constexpr (!SPLIT) l[1] *= fac;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e) O[c][e] *= fac;
      m = grown ? mt : m;
    }
    return m == -INFINITY ? 0.0f : m * p.scale_log2e;
  };
  // Probabilities of the quarter k of a tile's keys and, in fp32, their sum.  SPLIT: hi has their upper 16 bits and lo what that leaves, so that what meets V is within 2^-16 of them;
  // else hi is rounded to bf16 (2^-8) and the sum is of what was rounded.
  struct Probs { bf16x8 hi, lo; };
  auto quarter = [&](const Scores& S, int k, float ref) {
    uintx4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float x[2];
#pragma unroll
      for (int f = 0; f < 2; ++f) x[f] = __builtin_amdgcn_exp2f(__builtin_fmaf(S.u[k >> 1][8 * (k & 1) + 2 * e + f], p.scale_log2e, -ref));
      if constexpr (SPLIT) {
        const unsigned b0 = __builtin_bit_cast(unsigned, x[0]), b1 = __builtin_bit_cast(unsigned, x[1]);
        l[0] += x[0] + x[1];
        hi[e] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
        const bf16x2 left = {(__bf16)(x[0] - __builtin_bit_cast(float, b0 & 0xffff0000u)), (__bf16)(x[1] - __builtin_bit_cast(float, b1 & 0xffff0000u))};
        lo[e] = __builtin_bit_cast(unsigned, left);
      } else {
        const bf16x2 r = {(__bf16)x[0], (__bf16)x[1]};
        hi[e] = __builtin_bit_cast(unsigned, r);
        l[e & 1] = __builtin_amdgcn_fdot2_f32_bf16(r, bf16x2{(__bf16)1.0f, (__bf16)1.0f}, l[e & 1], false);
      }
    }
    return Probs{__builtin_bit_cast(bf16x8, hi), __builtin_bit_cast(bf16x8, lo)};
  };
  unsigned atK = base, atV = baseV;              // the tile of K whose scores come next, the tile of V
  // Tile s, whose scores are in S; those of the next one go to N.
  auto tile_step = [&](int s, Scores& S, Scores& N) {
    wait_loads<(RING - 2) * 2 * LH>();
    __builtin_amdgcn_s_barrier();                // K of the next tile and V of this one are there, and nobody reads those before them any more
    issue_k(s + RING);
    issue_v(s + RING - 1);
    atK = atK == base + (RING - 1) * TILE ? base : atK + TILE;
    const int k0 = first + s * KT;
    if (sees(s) || sees(s + 1)) {                // or the scores that follow are of no tile, but none of them is looked at
      clear(N);
      const bool whole = whi <= k0 && wq >= k0 + KT - 1;
      const int from = lo - k0 - 8 * h, to = q - k0 - 8 * h;
      if (!whole)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int key = 32 * u + 16 * (e >> 3) + (e & 7);          // and k0 + 8 h
            S.u[u][e] = key < from || key > to ? -INFINITY : S.u[u][e];
            __builtin_amdgcn_sched_barrier(0);                         // one comparison at a time, or their results take the scalar registers
          }
      const float ref = raise(S);
      // Where some key is not seen by every query, a value that is not finite would reach those too, by a probability of zero: such values are left out
      // of the products and added to the results of the queries that see them.
      bool odd = false;
      if (!whole || again) {
        typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
        ushort2v most = {0, 0};
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const uintx4 bits = __builtin_bit_cast(uintx4, frag_v(atV, c, k)) & 0x7fff7fffu;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const unsigned w = bits[e];
              most = __builtin_elementwise_max(most, __builtin_bit_cast(ushort2v, w));
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        odd = most[0] >= 0x7f80 || most[1] >= 0x7f80;
      }
      odd = __builtin_amdgcn_ballot_w64(odd) != 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        bf16x8 v[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) v[c] = frag_v(atV, c, k);
        scores(N, atK, k * NS / 4, (k + 1) * NS / 4);
        const Probs P = quarter(S, k, ref);
        if (odd)
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              v[c][e] = fabsf((float)v[c][e]) < INFINITY ? v[c][e] : (__bf16)0.0f;
              __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
        for (int c = 0; c < NC; ++c) O[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[c], P.hi, O[c], 0, 0, 0);
        if constexpr (SPLIT)
#pragma unroll
          for (int c = 0; c < NC; ++c) O[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[c], P.lo, O[c], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (odd)
#pragma unroll 1
        for (int i = 0; i < KT; ++i) {
          const bool seen = k0 + i >= lo && k0 + i <= q;
          if (!__builtin_amdgcn_ballot_w64(seen)) continue;
          int half = h;
          asm volatile("" : "+v"(half));         // or the addresses below are worked out ahead of everything, and kept
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int r = 32 * c + 8 * (e >> 2) + 4 * half + (e & 3);
              const float v = (float)*(const __attribute__((address_space(3))) __bf16*)(size_t)(atV + r * 128 + (((i >> 3) ^ ((r >> 1) & 7)) * 16) + (i & 7) * 2);
              O[c][e] += seen && !(fabsf(v) < INFINITY) ? v : 0.0f;
              __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    atV = atV == baseV + (RING - 1) * TILE ? baseV : atV + TILE;
  };
  while (true) {
    toK = atK = base;
    toV = atV = baseV;
    m = -INFINITY;
    l[0] = l[1] = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) O[c][e] = 0.0f;
    int s0 = 0;
    asm volatile("" : "+s"(s0));                 // or the addresses of these are worked out ahead, and kept
    issue_k(s0);
#pragma unroll
    for (int s = 0; s < RING - 1; ++s) {
      issue_k(s0 + s + 1);
      issue_v(s0 + s);
    }
    Scores a, b;
    clear(a);
    wait_loads<(RING - 1) * 2 * LH>();
    __builtin_amdgcn_s_barrier();
    all_scores(a, atK);
#pragma unroll 1
    for (int s = 0; s < steps; s += 2) {
      tile_step(s, a, b);
      if (s + 1 < steps) tile_step(s + 1, b, a);
    }
    wait_loads<0>();                             // LDS is not to be written behind the workgroup's end
    if (again) break;
    // A value of V that is not finite and is seen by every query of a tile has been multiplied by a probability or by a part of one, which may be zero: the workgroup then
    // goes through the keys once more and looks at every tile's values.
    float most = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) most = __builtin_elementwise_maximum(most, fabsf(O[c][e]));
    const bool lost = __builtin_amdgcn_ballot_w64(!(most < INFINITY)) != 0;
    if (lane == 0) lows[wave] = lost;
    __syncthreads();
    int any = lows[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) any |= lows[w];
    if (!__builtin_amdgcn_readfirstlane(any)) break;
    again = true;
  }
  const float half = l[0] + l[1];
  const auto halves = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, half), __builtin_bit_cast(unsigned, half), false, false);
  const unsigned half0 = halves[0], half1 = halves[1];
  const float inv = 1.0f / (__builtin_bit_cast(float, half0) + __builtin_bit_cast(float, half1));
  if (lo > q) return;
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int r = 32 * c + 8 * (e >> 2) + 4 * h + (e & 3);
      if (r < p.dh) ((__bf16*)p.C)[((long long)head * p.dh + r) * p.ldc + q] = (__bf16)(O[c][e] * inv);
    }
}

static void launch_attention_bf16(strp_ctx* ctx, AttnP p) {
  p.near = p.dh % 8 == 0 && 64 * p.ldk < (1LL << 31) && 64 * p.ldv < (1LL << 31);
  const auto go = [&](auto kernel, int bq, int threads) {
    p.tiles = (int)((p.T + bq - 1) / bq);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(p.tiles * p.heads)), dim3(threads), 0, ctx->stream, p);
  };
  // three workgroups of 64 channels on a CU, two of 96 or 128: what its 160 KB of LDS and its registers hold.  (With the probabilities in two terms, 64 channels and Q in registers it
  // would be two: 302 us, not 271, for 32 heads over 8 x 2048 tokens.)  Two tiles of K and of V in LDS or three: the same within 1 %.
  const auto by_width = [&](auto split) {
    constexpr bool SPLIT = decltype(split)::value;
    if (p.dh <= 64) go(attention_bf16_kernel<64, 4, SPLIT ? 2 : 3, 3, SPLIT>, 128, 256);
    else if (p.dh <= 96) go(attention_bf16_kernel<96, 4, 2, 2, SPLIT>, 128, 256);
    else go(attention_bf16_kernel<128, 4, 2, 2, SPLIT>, 128, 256);
  };
  if (ctx->precision == STRP_PREC_SPLIT) by_width(std::true_type());
  else by_width(std::false_type());
}

static void launch_attention_f32(strp_ctx* ctx, AttnP p) {
  p.tiles = (int)((p.T + 63) / 64);
  const dim3 grid((unsigned)(p.tiles * p.heads)), block(256);
  if (p.dh <= 64) hipLaunchKernelGGL((attention_f32_kernel<64>), grid, block, 0, ctx->stream, p);
  else if (p.dh <= 96) hipLaunchKernelGGL((attention_f32_kernel<96>), grid, block, 0, ctx->stream, p);
  else hipLaunchKernelGGL((attention_f32_kernel<128>), grid, block, 0, ctx->stream, p);
}

}  // namespace strp

using namespace strp;

extern "C" strp_status strp_attention(strp_ctx* ctx, const strp_attention_in* in) {
  if (!ctx) return STRP_EINVAL;
  if (!in || !in->Q || !in->K || !in->V || !in->C) return fail(ctx, STRP_EINVAL, "attention: null Q, K, V or C");
  if (!known_dtype(in->dtype)) return fail(ctx, STRP_EINVAL, "attention: unknown dtype");
  if (in->heads <= 0 || in->kv_heads <= 0 || in->d_head <= 0 || in->T <= 0) return fail(ctx, STRP_EINVAL, "attention: heads, kv_heads, d_head and T must be positive");
  if (in->d_head > 128) return fail(ctx, STRP_EINVAL, "attention: d_head above 128");
  if (in->heads > 65535) return fail(ctx, STRP_EINVAL, "attention: more than 65535 heads");
  if (!in->kv_of_head && in->heads % in->kv_heads) return fail(ctx, STRP_EINVAL, "attention: kv_heads does not divide heads and kv_of_head is null");
  if (in->n_seq < 0 || (in->seq_start ? in->n_seq < 1 : in->n_seq != 0)) return fail(ctx, STRP_EINVAL, "attention: seq_start needs n_seq > 0, no seq_start n_seq = 0");
  // the kernels multiply by scale log2(e)
  if (!(in->scale > 0.0f) || !(in->scale <= 2.0e38f)) return fail(ctx, STRP_EINVAL, "attention: scale must be positive and at most 2e38");
  if (!token_ld(in->ldq, in->T) || !token_ld(in->ldk, in->T) || !token_ld(in->ldv, in->T) || !token_ld(in->ldc, in->T))
    return fail(ctx, STRP_EINVAL, "attention: leading dimensions must be multiples of 8 and not below T");
  if (!ptr16(in->Q) || !ptr16(in->K) || !ptr16(in->V) || !ptr16(in->C)) return fail(ctx, STRP_EINVAL, "attention: Q, K, V or C not 16-byte aligned");
  if ((in->T + 63) / 64 * in->heads > MAX_TILES) return fail(ctx, STRP_EINVAL, "attention: tiles of 64 tokens of all heads, more than a launch holds");
  OnDevice on(ctx);
  if (!on.ok()) return fail(ctx, STRP_EHIP, "attention: device %d cannot be made current", ctx->device);
  AttnP p{in->Q, in->K, in->V, in->C, in->seq_start, in->kv_of_head, in->heads, in->kv_heads, in->heads / in->kv_heads, in->d_head, in->n_seq,
          0, in->T, in->ldq, in->ldk, in->ldv, in->ldc, in->scale * 1.44269504088896341f, 0};
  if (p.group == 0) p.group = 1;
  // the lengths are on the device: the operations of one sequence of all tokens
  const double T = (double)in->T;
  ProfScope ps(ctx, "attention", 2.0 * in->heads * in->d_head * T * (T + 1.0), bytes_of(in->dtype) * T * in->d_head * 2.0 * (in->heads + in->kv_heads));
  if (in->dtype == STRP_BF16) launch_attention_bf16(ctx, p);
  else launch_attention_f32(ctx, p);
  STRP_HIP(ctx, hipGetLastError());
  return STRP_OK;
}
