// Attention of new tokens over a paged cache in bf16, 128 rows at a time: chunks of prompts.
//
// S = K Q^T and O = V^T P by v_mfma_f32_32x32x16_bf16.  A workgroup has 128 rows (heads of a group by new tokens), each of its wavefronts 32, and goes through the keys 64
// at a time (of 4 bits 32); their rows of K and of V lie in LDS as in their pages, the chunks of 16 bytes of a row in an order that depends on the row, so that what is read at
// once lies in different banks.  A row is a lane's: S has the keys 8 (e / 4) + 4 (lane / 32) + e % 4 in its registers e, and where the fragments of V, read turned,
// have the keys in that order too, eight registers of P are a second operand of V^T P as they are.  The scores of the next keys are multiplied beside the softmax of these.
// Bound by the vector unit and the matrix cores, either busy half of the time: 1024 tokens of 32 heads of 128 (8 of keys) on 30000 keys 670-705 TFLOP/s, on 6000 560-570; 4 bits 357-375.
//
// Work is counted in units of so many keys of one tile, and every workgroup has as many as any other.  Tile i of e sees about as many keys as it leaves to tile e - 1 - i: tiles
// are taken in such pairs, which are all given the same number of units, so that nobody has to add up the tiles before his own.
#pragma once

#include "cache_attention.h"

#include <type_traits>

namespace strp {

__device__ const unsigned cache_zero_chunk[4] = {0u, 0u, 0u, 0u};

// KT: keys of a unit, fewer of 4 bits for the registers
template <int W, bool Q4>
struct Wide {
  static constexpr int DHP = 16 * W, PITCH = 2 * DHP, KT = Q4 ? 32 : 64, TILE = KT * PITCH, RING = 2, BYTES = 2 * RING * TILE > 4 * MAX_CACHE_HEADS ? 2 * RING * TILE : 4 * MAX_CACHE_HEADS;
};

// Whole numbers of 4 bits, two channels a byte, as bf16 in the channels' order.
__device__ __forceinline__ uintx4 numbers_of(unsigned x) {
  const unsigned even = x & 0x0f0f0f0fu, odd = (x >> 4) & 0x0f0f0f0fu;
  uintx4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r[i] = pick(__builtin_bit_cast(unsigned, (float)((even >> (8 * i)) & 255u)), __builtin_bit_cast(unsigned, (float)((odd >> (8 * i)) & 255u)), HIGHS);
  return r;
}

// Q4: keys and values come by way of registers, as whole numbers in bf16; lowest and step of K enter the scores, those of V the probabilities, in fp32.
template <int W, bool SPLIT, bool Q4>
__device__ __forceinline__ void wide_share(const RowsP& p, const Heads& heads, unsigned char* smem, unsigned block) {
  typedef Wide<W, Q4> Z;
  constexpr int NC = Z::DHP / 32, NS = Z::DHP / 16, KT = Z::KT, U = KT / 32, KEYS = KT / 4, PITCH = Z::PITCH, TILE = Z::TILE, LOADS = TILE / 4096;      // LOADS: KBs of a tile that a wavefront moves
  constexpr int CHUNKS = PITCH / 16, EACH = 64 / CHUNKS;                   // chunks of a row, rows of a KB
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, l32 = lane & 31;
  const Pages& c = p.c;
  const int dh = c.dh;
  const int worker = (int)(block & 7) * (WORKERS >> 3) + (int)(block >> 3);      // neighbours in the work are neighbours on an XCD

  struct Rows {                            // the rows of a sequence that share a key-value head
    int n, past, cap, group, rows, tiles, paired;
    long long pair, units;                 // units of a pair of tiles, of all
    __device__ __forceinline__ int units_of(int tile) const {
      const int token = min((tile * WIDE + WIDE - 1) / group, n - 1);
      return (min(past + token, cap - 1) + KT) / KT;
    }
  };
  auto rows_of = [&](int n, int past, int group) {
    Rows r{n, past, c.cap, group, n * group, 0, 0, 0, 0};
    if (r.rows <= WIDE_FROM) return r;
    r.tiles = (r.rows + WIDE - 1) / WIDE;
    r.paired = r.tiles & ~1;
    const int last = r.units_of(r.tiles - 1);
    if (r.paired) {
      const long long both = 2LL * past + 2 + ((r.paired - 1) * WIDE + 2 * WIDE - 2) / group;      // no fewer keys than the two tiles of a pair see together
      r.pair = min((both + 2 * (KT - 1)) / KT, 2LL * last);
    }
    r.units = (r.paired / 2) * r.pair + (r.tiles & 1 ? last : 0);
    return r;
  };
  struct Seq { int begin, n, past; long long units; };
  auto sequence = [&](int s) {
    Seq q;
    q.begin = seq_begin(c, s);
    q.n = max(seq_begin(c, s + 1) - q.begin, 0);
    q.past = seq_past(c, s);
    q.units = 0;
    if (q.n) {
      if (!heads.first) q.units = c.kv_heads * rows_of(q.n, q.past, heads.group).units;
      else
        for (int kv = 0; kv < c.kv_heads; ++kv) q.units += rows_of(q.n, q.past, heads.of(kv)).units;
    }
    return q;
  };
  const int each = (c.n_seq + 63) / 64;
  long long mine = 0;
  for (int i = 0; i < each; ++i)
    if (lane * each + i < c.n_seq) mine += sequence(lane * each + i).units;
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long x = __shfl_up(upto, o, 64);
    upto += lane >= o ? x : 0;
  }
  const long long total = uniform(__shfl(upto, 63, 64));
  long long per = (total + WORKERS - 1) / WORKERS;
  per = per < p.wide_least ? p.wide_least : per;
  long long u = worker * per;
  const long long u1 = u + per < total ? u + per : total;
  if (tid == 0) p.wide_parts[worker] = 0;
  if (u >= u1) return;
  const unsigned long long holds = __builtin_amdgcn_ballot_w64(upto - mine <= u && u < upto);
  const int holder = __builtin_ctzll(holds);
  int s = __builtin_amdgcn_readfirstlane(holder * each);
  long long base = uniform(__shfl(upto - mine, holder, 64));
  auto same = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  auto uniform_sequence = [&] {
    const Seq x = sequence(s);
    return Seq{same(x.begin), same(x.n), same(x.past), uniform(x.units)};
  };
  Seq q = uniform_sequence();

  const unsigned ldsK = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem, ldsV = ldsK + Z::RING * TILE;
  // a wavefront moves KEYS rows of a tile, EACH of them at a time: lane l has chunk l % CHUNKS of row l / CHUNKS of them
  auto order_k = [](int row) { return (row / (256 / PITCH)) & (CHUNKS - 1); };
  auto order_v = [](int row) { return PITCH == 256 ? (row & 3) << 2 : PITCH == 128 ? ((row >> 1) & 1) << 2 : 0; };
  const bool full = 2 * dh == PITCH;
  __shared__ __attribute__((aligned(16))) float2 scales[Q4 ? 2 : 1][Q4 ? 3 : 1][Q4 ? KT : 1];      // of K and V, three units: some wavefronts are a unit ahead of others
  __shared__ int not_finite[Q4 ? 3 : 1][4];                                // of V's, a bit for a key
  // fragments of K: key l32 (+ 32 u), chunk 2 d + h; of V: keys 16 k + 4 h + (lane % 16) / 4 (+ 8), the 16 channels of the lane's group
  const int kr = (lane & 15) >> 2;
  const unsigned offK = (unsigned)(l32 * PITCH + ((h ^ order_k(l32)) * 16));
  const unsigned offV = (unsigned)((4 * h + kr) * PITCH + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ order_v(kr)) * 16) + (lane & 1) * 8);
  auto frag_k = [&](unsigned at, int d, int t) { return *(const __attribute__((address_space(3))) bf16x8*)(size_t)(at + (offK ^ (unsigned)(32 * d)) + 32 * PITCH * t); };
  auto frag_v = [&](unsigned at, int ch, int k) {
    const unsigned a = at + (offV ^ (unsigned)(64 * ch)) + 16 * PITCH * k;
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(read_turned(a), read_turned(a + 8 * PITCH), 0, 1, 2, 3, 4, 5, 6, 7));
  };

  while (true) {
    while (u >= base + q.units) {
      base += q.units;
      ++s;
      q = uniform_sequence();
    }
    // ---- a segment: units b0 .. b1 of one tile of rows ----
    long long rel = u - base;
    int kv = 0;
    Rows rw;
    if (!heads.first) {
      rw = rows_of(q.n, q.past, heads.group);
      kv = (int)(rel / rw.units);
      rel -= kv * rw.units;
    } else {
      for (;; ++kv) {
        rw = rows_of(q.n, q.past, same(heads.of(kv)));
        if (rel < rw.units) break;
        rel -= rw.units;
      }
    }
    int tile = rw.tiles - 1, b0;
    const long long single = (rw.paired / 2) * rw.pair;
    if (rel >= single) {
      b0 = (int)(rel - single);
    } else {
      const int i = (int)(rel / rw.pair), j = (int)(rel - i * rw.pair), first = rw.units_of(i), second = rw.units_of(rw.paired - 1 - i);
      tile = j < first ? i : rw.paired - 1 - i;
      b0 = j < first ? j : j - first;
      if (j >= first + second) {           // what the pair has been given beyond its units
        u += rw.pair - j;
        if (u >= u1) return;
        continue;
      }
    }
    const int units = rw.units_of(tile), b1 = units - b0 < u1 - u ? units : b0 + (int)(u1 - u), steps = b1 - b0;
    const int rows = min(WIDE, rw.rows - tile * WIDE), r = wave * 32 + l32, at = tile * WIDE + min(r, rows - 1), token = at / rw.group, in_group = at - token * rw.group;
    const int head = heads.head(kv, in_group), keys = min(q.past + q.n, c.cap);
    const int see = min(q.past + token, keys - 1);                         // the row's last key
    // of the wavefront's rows: the last key that all see, that any sees (none, where it has no rows)
    const int see_all = same(min(q.past + (tile * WIDE + min(wave * 32, rows - 1)) / rw.group, keys - 1));
    const int see_any = wave * 32 < rows ? same(min(q.past + (tile * WIDE + min(wave * 32 + 31, rows - 1)) / rw.group, keys - 1)) : -1;
    bf16x8 qf[NS];
    {
      const __bf16* Q = (const __bf16*)p.Q + (long long)head * dh * p.ldq + q.begin + token;
      int width = dh, half = h;
      asm volatile("" : "+s"(width), "+v"(half));                          // what this works out is not worth registers for the rest of the kernel
#pragma unroll
      for (int d = 0; d < NS; ++d)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int ch = 16 * d + 8 * half + e;
          qf[d][e] = Q[(long long)(ch < width ? ch : 0) * p.ldq];
        }
      __builtin_amdgcn_sched_barrier(0);                                   // all of them asked for before any is waited for
#pragma unroll
      for (int d = 0; d < NS; ++d)
#pragma unroll
        for (int e = 0; e < 8; ++e) qf[d][e] = 16 * d + 8 * half + e < width ? qf[d][e] : (__bf16)0.0f;
    }
    float qsum = 0.0f;
    if constexpr (Q4) {
#pragma unroll
      for (int d = 0; d < NS; ++d)
#pragma unroll
        for (int e = 0; e < 8; ++e) qsum += (float)qf[d][e];
      qsum = both_32(qsum, true);
    }

    // pages of the wavefront's keys of a unit: lane l has that of unit bt + l
    const int32_t* table = c.table + (long long)s * c.ld_table;
    const int in_page = (1 << c.page_log2) - 1;
    int ids = 0, bt = 0;
    auto look_up = [&](int b) {
      bt = b;
      ids = clamped(table[min((int)(((long long)(b + lane) * KT + wave * KEYS) >> c.page_log2), c.ld_table - 1)], 0, c.pages - 1);
    };
    auto issue = [&](const void* pool, long long row, unsigned to, bool of_k) {
      const char* from = (const char*)pool + row * (2 * dh);
      to += (unsigned)wave * (KEYS * PITCH);
      int mine = lane, width = dh;
      asm volatile("" : "+v"(mine), "+s"(width));        // worked out each time, for the registers
      auto piece = [&](int i) { return mine / CHUNKS + EACH * i; };      // its row
      auto chunk_of = [&](int row) { return (mine % CHUNKS) ^ (of_k ? order_k(row) : order_v(row)); };
      if (full) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) copy_to_lds_from(from, (unsigned)(piece(i) * PITCH + chunk_of(piece(i)) * 16), to + 1024 * i);
      } else {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const int row = piece(i), chunk = chunk_of(row);
          copy_to_lds(8 * chunk < width ? (const void*)(from + (unsigned)(row * width + chunk * 8) * 2u) : (const void*)cache_zero_chunk, to + 1024 * i);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    unsigned toK, toV, atK, atV;           // where the next tile goes, and is read
    long long next_row = 0;
    // 4 bits: a lane has an eighth of the channels of a key of K and of one of V (heads of 32: a fourth, or nothing), and K's scales of that key or V's or nothing
    constexpr int PARTS = 64 / KEYS, DW = W >= 4 ? W / 4 : 1;
    struct Packed { unsigned k[DW], v[DW]; float2 scale; };
    auto page_of = [&](int b) {            // units in their order
      if (b - bt == 64) look_up(b);
      const int page = __builtin_amdgcn_readlane(ids, b - bt);
      return (((long long)page * c.kv_heads + kv) << c.page_log2) + ((b * KT + wave * KEYS) & in_page);
    };
    auto ask_packed = [&](long long k_row, long long v_row) {
      Packed x;
      int mine = lane, width = dh;
      asm volatile("" : "+v"(mine), "+s"(width));        // worked out each time, for the registers
      const int key = mine / PARTS, part = mine % PARTS;
      const auto gk = opaque((const char*)p.K + k_row * (dh / 2)), gv = opaque((const char*)p.V + v_row * (dh / 2));
#pragma unroll
      for (int j = 0; j < DW; ++j) {
        const int chunk = part * DW + j;
        const unsigned off = (unsigned)(key * (width / 2) + (8 * chunk < width ? 4 * chunk : 0));      // (channels that are not there meet queries of zero, or nobody)
        x.k[j] = *(Global<unsigned>)(gk + off);
        x.v[j] = *(Global<unsigned>)(gv + off);
      }
      const auto gs = (part & 1 ? opaque((const float2*)p.sV + v_row) : opaque((const float2*)p.sK + k_row)) + 8u * (unsigned)key;
      x.scale = float2{((Global<float>)gs)[0], ((Global<float>)gs)[1]};
      return x;
    };
    // K of the unit that goes to slot ks of three, V of that before it
    auto put_packed = [&](const Packed& x, unsigned to_k, unsigned to_v, int k_unit) {
      int mine = lane;
      asm volatile("" : "+v"(mine));
      const int key = mine / PARTS, part = mine % PARTS, row = wave * KEYS + key;
#pragma unroll
      for (int j = 0; j < DW; ++j) {
        const int chunk = part * DW + j;
        if (PARTS * DW > CHUNKS && chunk >= CHUNKS) continue;
        *(__attribute__((address_space(3))) uintx4*)(size_t)(to_k + row * PITCH + ((chunk ^ order_k(row)) * 16)) = numbers_of(x.k[j]);
        *(__attribute__((address_space(3))) uintx4*)(size_t)(to_v + row * PITCH + ((chunk ^ order_v(row)) * 16)) = numbers_of(x.v[j]);
      }
      // scales of V that are not finite would reach rows that do not see their key, by a probability of zero: they are looked at by themselves
      const bool bad = part == 1 && !(fabsf(x.scale.x) < INFINITY && fabsf(x.scale.y) < INFINITY);
      const unsigned long long which = __builtin_amdgcn_ballot_w64(bad);
      const int k_slot = k_unit % 3, v_slot = (k_unit + 2) % 3;
      if (part < 2) scales[part][part ? v_slot : k_slot][row] = bad ? float2{0.0f, 0.0f} : x.scale;
      if (lane == 0) {
        int bits = 0;
        if (which)
          for (int i = 0; i < KEYS; ++i) bits |= (int)(which >> (PARTS * i + 1) & 1) << i;
        not_finite[v_slot][wave] = bits;
      }
    };
    auto ahead = [&](unsigned& x, unsigned from) { x = x == from + (Z::RING - 1) * TILE ? from : x + TILE; };
    auto issue_k = [&](int b) {
      next_row = page_of(b);
      issue(p.K, next_row, toK, true);
      ahead(toK, ldsK);
    };
    auto issue_v = [&](long long row) {
      issue(p.V, row, toV, false);
      ahead(toV, ldsV);
    };

    floatx16 O[NC];
    float m, l[2], lowest;                 // lowest: the sum of p lowest, of 4 bits
    bool again = false;
    struct Scores { floatx16 u[U]; };
    auto clear = [&](Scores& S) {
#pragma unroll
      for (int t = 0; t < U; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) S.u[t][e] = 0.0f;
    };
    auto scores = [&](Scores& S, unsigned from, int d0, int d1) {
#pragma unroll
      for (int d = d0; d < d1; ++d)
#pragma unroll
        for (int t = 0; t < U; ++t) S.u[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_k(from, d, t), qf[d], S.u[t], 0, 0, 0);
    };
    // the running maximum with a tile's scores, what is held rescaled to it; returns what is to be taken from a score in powers of two
    auto raise = [&](Scores& S) {
      float mt = m;
#pragma unroll
      for (int t = 0; t < U; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) mt = __builtin_elementwise_maximum(mt, S.u[t][e]);
      mt = both_32(mt, false);
      // what a row holds stays as it is until its maximum has grown past 2^8 times: probabilities of up to 256 are as good as those below 1
      const bool grown = !((mt - m) * p.scale_log2e <= 8.0f || mt == -INFINITY);
      if (__builtin_amdgcn_ballot_w64(grown)) {
        const float fac = grown ? between<true>(m, mt, p.scale_log2e) : 1.0f;
        l[0] *= fac;
        if constexpr (!SPLIT || Q4) l[1] *= fac;
        if constexpr (Q4) lowest *= fac;
#pragma unroll
        for (int ch = 0; ch < NC; ++ch)
#pragma unroll
          for (int e = 0; e < 16; ++e) O[ch][e] *= fac;
        m = grown ? mt : m;
      }
      const float ref = m == -INFINITY ? 0.0f : m, ref_log2 = ref * p.scale_log2e;
      const bool far = !(fabsf(ref_log2) < FAR);
      if (__builtin_amdgcn_ballot_w64(far))
#pragma unroll
        for (int t = 0; t < U; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) S.u[t][e] -= far ? ref : 0.0f;
      return far ? 0.0f : ref_log2;
    };
    // Probabilities of the quarter k of a tile's keys and, in fp32, their sum.  SPLIT: hi has their upper 16 bits and lo what that leaves, together within 2^-16 of them;
    // else hi is rounded to bf16 and the sum is of what was rounded.
    struct Probs { bf16x8 hi, lo; };
    auto quarter = [&](const Scores& S, int k, float ref, int b) {
      uintx4 hi, lo;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x[2];
#pragma unroll
        for (int f = 0; f < 2; ++f) x[f] = __builtin_amdgcn_exp2f(__builtin_fmaf(S.u[k >> 1][8 * (k & 1) + 2 * e + f], p.scale_log2e, -ref));
        if constexpr (Q4) {
          l[0] += x[0] + x[1];
          const int key = 16 * k + 8 * (e >> 1) + 2 * (e & 1);             // and 4 h: the first of the two
          const floatx4 s = *(const floatx4*)&scales[1][b % 3][key + 4 * h];
#pragma unroll
          for (int f = 0; f < 2; ++f) {
            lowest = __builtin_fmaf(x[f], s[2 * f], lowest);
            x[f] *= s[2 * f + 1];
          }
        }
        if constexpr (SPLIT) {
          const unsigned x0 = __builtin_bit_cast(unsigned, x[0]), x1 = __builtin_bit_cast(unsigned, x[1]);
          if constexpr (!Q4) l[0] += x[0] + x[1];
          hi[e] = pick(x0, x1, HIGHS);
          const bf16x2 left = {(__bf16)(x[0] - __builtin_bit_cast(float, x0 & 0xffff0000u)), (__bf16)(x[1] - __builtin_bit_cast(float, x1 & 0xffff0000u))};
          lo[e] = __builtin_bit_cast(unsigned, left);
        } else {
          const bf16x2 one = {(__bf16)x[0], (__bf16)x[1]};
          hi[e] = __builtin_bit_cast(unsigned, one);
          if constexpr (!Q4) l[e & 1] = __builtin_amdgcn_fdot2_f32_bf16(one, bf16x2{(__bf16)1.0f, (__bf16)1.0f}, l[e & 1], false);
        }
      }
      return Probs{__builtin_bit_cast(bf16x8, hi), __builtin_bit_cast(bf16x8, lo)};
    };
    [[maybe_unused]] Packed pending;       // of 4 bits: K two units ahead and V one, on their way for a unit already
    // Unit b, whose scores are in S; those of the next one go to N.
    auto unit = [&](int b, Scores& S, Scores& N) {
      if constexpr (Q4) {
        __syncthreads();
      } else {
        wait_loads<0>();
        __builtin_amdgcn_s_barrier();      // K of the next unit and V of this one are there, and nobody reads those before them any more
      }
      [[maybe_unused]] Packed packed;
      const long long row = next_row;      // of unit b + 1, of 4 bits b + 2
      if constexpr (Q4) {
        next_row = page_of(b + 3);         // (what lies behind the last unit is asked for too, and nobody looks at it: a condition here would cost registers)
        packed = ask_packed(next_row, row);
      } else if (b + 1 < b1) {
        if (b + 2 < b1) issue_k(b + 2);
        else ahead(toK, ldsK);
        issue_v(row);
      }
      ahead(atK, ldsK);
      const int k0 = b * KT;
      if (k0 <= see_any) {
        clear(N);
        const bool whole = k0 + KT - 1 <= see_all;
        const int to = see - k0 - 4 * h;
        if constexpr (Q4)
#pragma unroll
          for (int t = 0; t < U; ++t)
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
              const floatx4 s = *(const floatx4*)&scales[0][b % 3][32 * t + 8 * (e >> 2) + 4 * h + (e & 3)];
#pragma unroll
              for (int f = 0; f < 2; ++f) S.u[t][e + f] = __builtin_fmaf(S.u[t][e + f], s[2 * f + 1], qsum * s[2 * f]);
              __builtin_amdgcn_sched_barrier(0);
            }
        if (!whole)
#pragma unroll
          for (int t = 0; t < U; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              S.u[t][e] = 32 * t + 8 * (e >> 2) + (e & 3) > to ? -INFINITY : S.u[t][e];
              __builtin_amdgcn_sched_barrier(0);       // one comparison at a time, or their results take the scalar registers
            }
        // products first: while they go on, another wavefront has the vector unit (4 bits: 317 us without, 299 for 1024 tokens on 6000 keys; bf16 the same; with a unit more on its way 292)
        __builtin_amdgcn_s_setprio(0);
        const float ref = raise(S);
        __builtin_amdgcn_s_setprio(1);
        // Where some key is not seen by every row, a value that is not finite would reach those too, by a probability of zero: such values are left out
        // of the products and added to the results of the rows that see them.
        bool odd = false;
        if (!Q4 && (!whole || again)) {
          typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
          ushort2v most = {0, 0};
#pragma unroll
          for (int k = 0; k < 2 * U; ++k)
#pragma unroll
            for (int ch = 0; ch < NC; ++ch) {
              const uintx4 bits = __builtin_bit_cast(uintx4, frag_v(atV, ch, k)) & 0x7fff7fffu;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const unsigned w = bits[e];
                most = __builtin_elementwise_max(most, __builtin_bit_cast(ushort2v, w));
              }
              __builtin_amdgcn_sched_barrier(0);
            }
          odd = most[0] >= 0x7f80 || most[1] >= 0x7f80;
        }
        odd = !Q4 && __builtin_amdgcn_ballot_w64(odd) != 0;
#pragma unroll
        for (int k = 0; k < 2 * U; ++k) {
          bf16x8 v[NC];
#pragma unroll
          for (int ch = 0; ch < NC; ++ch) v[ch] = frag_v(atV, ch, k);
          scores(N, atK, k * NS / (2 * U), (k + 1) * NS / (2 * U));
          __builtin_amdgcn_s_setprio(0);
          const Probs P = quarter(S, k, ref, b);
          __builtin_amdgcn_s_setprio(1);
          if (odd)
#pragma unroll
            for (int ch = 0; ch < NC; ++ch)
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                v[ch][e] = fabsf((float)v[ch][e]) < INFINITY ? v[ch][e] : (__bf16)0.0f;
                __builtin_amdgcn_sched_barrier(0);
              }
#pragma unroll
          for (int ch = 0; ch < NC; ++ch) O[ch] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[ch], P.hi, O[ch], 0, 0, 0);
          if constexpr (SPLIT)
#pragma unroll
            for (int ch = 0; ch < NC; ++ch) O[ch] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[ch], P.lo, O[ch], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (Q4) {
          const int slot = b % 3;
          const int any = __builtin_amdgcn_readfirstlane(not_finite[slot][0] | not_finite[slot][1] | not_finite[slot][2] | not_finite[slot][3]);
          if (any)
#pragma unroll 1
            for (int i = 0; i < KT; ++i)
              if (not_finite[slot][i / KEYS] >> (i % KEYS) & 1) lowest = k0 + i <= see ? __builtin_nanf("") : lowest;
        }
        if (odd)
#pragma unroll 1
          for (int i = 0; i < KT && k0 + i <= see_any; ++i) {
            const bool seen = k0 + i <= see;
            int half = h;
            asm volatile("" : "+v"(half));             // or the addresses below are worked out ahead of everything, and kept
#pragma unroll
            for (int ch = 0; ch < NC; ++ch)
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const int x = 32 * ch + 8 * (e >> 2) + 4 * half + (e & 3);
                const float v = (float)*(const __attribute__((address_space(3))) __bf16*)(size_t)(atV + i * PITCH + (((x >> 3) ^ order_v(i)) * 16) + (x & 7) * 2);
                O[ch][e] += seen && !(fabsf(v) < INFINITY) ? v : 0.0f;
                __builtin_amdgcn_sched_barrier(0);
              }
          }
      }
      if constexpr (Q4)
        if (b + 1 < b1) {
          put_packed(pending, toK, toV, b + 2);
          ahead(toK, ldsK);
          ahead(toV, ldsV);
        }
      if constexpr (Q4) pending = packed;
      ahead(atV, ldsV);
    };
    int* lost_of = (int*)smem;             // between the passes, of the four wavefronts
    while (true) {
      toK = atK = ldsK;
      toV = atV = ldsV;
      m = -INFINITY;
      l[0] = l[1] = lowest = 0.0f;
#pragma unroll
      for (int ch = 0; ch < NC; ++ch)
#pragma unroll
        for (int e = 0; e < 16; ++e) O[ch][e] = 0.0f;
      __syncthreads();                     // nobody reads the segment before any more
      look_up(b0);
      // (behind the last unit: pages that lie in the cache, for nobody)
      Scores a, b;
      clear(a);
      if constexpr (Q4) {
        const long long row = page_of(b0), second = page_of(b0 + 1);
        next_row = page_of(b0 + 2);
        const Packed x = ask_packed(row, row), y = ask_packed(second, row);
        pending = ask_packed(next_row, second);
        put_packed(x, toK, toV, b0 + 3);                 // (its V comes again with the next; the slots of three units further are its own)
        ahead(toK, ldsK);
        __syncthreads();
        put_packed(y, toK, toV, b0 + 1);
        ahead(toK, ldsK);
        ahead(toV, ldsV);
        __syncthreads();
      } else {
        issue_k(b0);
        const long long row = next_row;
        issue_k(b0 + 1);
        issue_v(row);
        wait_loads<2 * LOADS>();
        __builtin_amdgcn_s_barrier();
      }
#pragma unroll
      for (int d = 0; d < NS; d += 2) {
        scores(a, atK, d, d + 2);
        __builtin_amdgcn_sched_barrier(0); // not every fragment at once, for the registers
      }
#pragma unroll 1
      for (int i = b0; i < b1; i += 2) {
        unit(i, a, b);
        if (i + 1 < b1) unit(i + 1, b, a);
      }
      if constexpr (Q4) break;
      wait_loads<0>();                     // LDS is not to be written behind this
      if (again) break;
      // A value of V that is not finite and is seen by every row of a tile has been multiplied by a probability or by a part of one, which may be zero: the workgroup then
      // goes through the keys once more and looks at every tile's values.
      float most = 0.0f;
#pragma unroll
      for (int ch = 0; ch < NC; ++ch)
#pragma unroll
        for (int e = 0; e < 16; ++e) most = __builtin_elementwise_maximum(most, fabsf(O[ch][e]));
      const bool lost = __builtin_amdgcn_ballot_w64(!(most < INFINITY)) != 0;
      __syncthreads();
      if (lane == 0) lost_of[wave] = lost;
      __syncthreads();
      if (!__builtin_amdgcn_readfirstlane(lost_of[0] | lost_of[1] | lost_of[2] | lost_of[3])) break;
      again = true;
    }
    const float sum = both_32(l[0] + l[1], true);
    if constexpr (Q4) {
      lowest = both_32(lowest, true);
#pragma unroll
      for (int ch = 0; ch < NC; ++ch)
#pragma unroll
        for (int e = 0; e < 16; ++e) O[ch][e] += lowest;
    }
    int width = dh, half = h;
    asm volatile("" : "+s"(width), "+v"(half));                            // what follows from these is worked out here, not kept from segment to segment
    const long long out = r < rows ? (long long)head * dh * p.ldc + q.begin + token : -1;
    if (b0 == 0 && b1 == units) {
      const float inv = 1.0f / sum;
      if (out >= 0)
#pragma unroll
        for (int ch = 0; ch < NC; ++ch)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int x = 32 * ch + 8 * (e >> 2) + 4 * half + (e & 3);
            if (x < width) ((__bf16*)p.C)[out + (long long)x * p.ldc] = (__bf16)(O[ch][e] * inv);
            __builtin_amdgcn_sched_barrier(0);
          }
    } else {
      const int slot = worker * 2 + (b0 == 0 ? 1 : 0);
      const float by = __builtin_amdgcn_exp2f(-left_over<true>(m, p.scale_log2e));      // parts are joined as if exponents were not rounded
      float* part = p.wide_part + (long long)slot * width * WIDE + r;
      if (wave * 32 < rows)
#pragma unroll
        for (int ch = 0; ch < NC; ++ch)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int x = 32 * ch + 8 * (e >> 2) + 4 * half + (e & 3);
            if (x < width) part[x * WIDE] = O[ch][e] * by;
            __builtin_amdgcn_sched_barrier(0);
          }
      if (h == 0) {
        p.wide_ml[slot * WIDE + r] = float2{m, sum * by};
        p.wide_off[slot * WIDE + r] = out;
      }
      // the workgroups from this one to that with the tile's last unit
      if (b0 == 0 && tid == 0) p.wide_parts[worker] = (int)((u + units - 1) / per) - worker + 1;
    }
    u += steps;
    if (u >= u1) return;
  }
}

// The parts of tiles that several workgroups had, in the order of the keys: a thread has a row, and every 32nd channel.
__device__ __forceinline__ void wide_join(const RowsP& p, int worker, int y) {
  const int parts = p.wide_parts[worker];
  if (parts == 0) return;
  const int row = threadIdx.x & (WIDE - 1), ch0 = 2 * y + (int)(threadIdx.x / WIDE), dh = p.c.dh;
  const int first = worker * 2 + 1;
  const long long to = p.wide_off[first * WIDE + row];
  if (to < 0) return;
  float m = -INFINITY, l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](auto count) {             // so many at a time
    constexpr int UN = decltype(count)::value;
    for (int i0 = 0; i0 < parts; i0 += UN) {
      float2 ml[UN];
      float x[UN][4];
#pragma unroll
      for (int k = 0; k < UN; ++k) {
        const int i = min(i0 + k, parts - 1), slot = i == 0 ? first : (worker + i) * 2;
        ml[k] = p.wide_ml[slot * WIDE + row];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[k][j] = p.wide_part[((long long)slot * dh + min(ch0 + 32 * j, dh - 1)) * WIDE + row];
      }
      float most = m;
#pragma unroll
      for (int k = 0; k < UN; ++k) most = i0 + k < parts ? __builtin_elementwise_maximum(most, ml[k].x) : most;
      const auto factor = [&](float of) { return of == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((of - most) * p.scale_log2e); };
      const float f = factor(m);
      m = most;
      l *= f;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] *= f;
#pragma unroll
      for (int k = 0; k < UN; ++k)
        if (i0 + k < parts) {
          const float g = factor(ml[k].x);
          l += g * ml[k].y;
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j] += g * x[k][j];
        }
    }
  };
  if (parts <= 4) add(std::integral_constant<int, 4>());
  else add(std::integral_constant<int, 8>());      // 81 parts: 22 us, 26 four at a time; two parts of 512 tiles: 23 us, 18 four at a time
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (ch0 + 32 * j < dh) ((__bf16*)p.C)[to + (long long)(ch0 + 32 * j) * p.ldc] = (__bf16)(o[j] / l);
}

}  // namespace strp
