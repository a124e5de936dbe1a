// Attention of single queries over pages in tiles of the matrix cores: over the paged cache of 8 bits, and over a prefix
// whose pages several sequences share (in any of the three forms of the cache) together with the sequences' own pages.
//
// The columns of a tile are queries of one key/value head: the query heads that share it, of one sequence or, for a
// prefix, of all rows of the group that shares the pages.  Per 16 x 16 x 32 instruction
//   scores  S[key, column]  = K[key, :] . Q[column, :]        operand A = 16 keys, operand B = 16 columns
//   output  O^T[d, column] += V^T[d, key] . P[key, column]    operand A = 16 features, operand B = P
// In the result of the first a lane has one column (lane % 16) and 4 keys, so the softmax's running maximum and sum are
// scalars of a lane; with the keys dealt out as below the probabilities are already the second product's operand B.
// Values of 8 bits go to bf16 exactly; the scales of K multiply the scores, those of V the probabilities, in fp32.
// For the second product a probability (times V's scale) is two bf16 numbers, the nearest and what that leaves: at most 2^-16
// of it is lost, and what is left of a result's error is its own rounding to bf16.  (The nearest alone, 2^-8: the error against
// 64 bits is 1.3 to 2.4 % larger over hundreds of tokens, 13 % over 37.  The second product twice costs 1 to 2 % where HBM
// bounds the kernel, with the append 64 sequences of 545 e4m3 tokens 70.0 -> 71.0 us, 128 of 16 to 2048 109.1 -> 110.0, and 10 %
// in wide tiles: 7, 40 and 1 rows of 64 heads on 8 behind some 7000 bf16 tokens 40.1 -> 44.2.)  In wide tiles over 8 bits it is
// the nearest alone: what V itself loses in 8 bits is 4 to 16 times as much, and both would take 41.2 us there instead of 37.2,
// for an error that is 0.2 % smaller.  The sum is that of the unrounded probabilities.
//
// A launch has up to two parts, the groups' prefixes and the rows' own pages, and a workgroup of 4 waves takes one
// (group, key/value head, block of columns, split of the pages) of either part:
//  * narrow, up to 16 columns: the waves take turns by chunks of 32 keys, from global memory straight to registers, and
//    their states (maximum, sum, output) are merged through LDS.  HBM bounds it.
//  * wide, 64 columns: each wave has 16 of them, and all see the same tiles of 64 keys, which the workgroup brings to bf16
//    and into LDS once.  What a tile takes in LDS accesses and softmax bounds it, not its bytes.
// Where a (row, head) has more than one state, they are written out in fp32 and a second launch merges them in order.  Short
// prefixes are no part of their own: every row's workgroup takes its prefix and then its own pages, and there are no states.
//
// Measured, the launches alone under a trace, medians of several processes (a 1 GiB read reaches 5.9 TB/s here): 40 heads, e4m3,
// 64 sequences of 545 tokens 67 to 70 us = 5.2 to 5.5 TB/s; int8, 128 of 16 to 2048 104 to 122 us = 4.8 to 5.6 (without a trace,
// from pass to pass and with the append, 109 to 110); 64 heads on 8, e4m3, 48 of 1024 to 4096 60 us = 4.9 (the pieces are
// unequal) and 4.8 for the states; int8, one of 65538 30 to 31 us = 4.4 and 4.7.  Shared: 64 rows of 40 heads behind 2048 bf16
// tokens, 16 to 256 of their own, 40 to 42 us = 5.1 TB/s and 5; 7, 40 and 1 rows of 64 heads on 8 behind some 7000 e4m3 tokens
// 35 to 36 us and 4.9, together 0.28 PFLOP/s (wide tiles).  The least call is 5 us.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kv_quant.h"

namespace ds {

constexpr int kTileThreads = 256, kTileWaves = 4;
constexpr int kWideCols = 64, kNarrowCols = 16;
constexpr int kWideKeys = 64;  // of a tile

struct TilePart {
  const int32_t* cu_rows;  // group i has the rows [cu_rows[i], cu_rows[i + 1]); null: row i
  const int32_t* lens;
  const int32_t* tables;
  int len_add, max_len, max_pages, groups;
  int blocks_x;            // key/value heads x blocks of columns
  int splits, pages_per_split;  // (0: up to so many pieces, by how unequal the sequences are)
  int first_state;         // states of this part's splits
  int wide;                // 64 columns a workgroup
  int solo;                // narrow: a key/value head for each wave
  int rank;                // longest groups first
};

struct TileArgs {
  TilePart part[2];
  int first_blocks;  // workgroups of part 0
  const uint16_t* q;
  int q_stride;
  const void *k, *v;
  const uint16_t *k_scale, *v_scale;
  int n_heads, n_kv_heads;
  int n_states;      // of a (row, head); 1: o is written
  float scale_log2e;
  uint16_t* o;
  float* partial;    // [row][head][state][output[HD], max, sum, states of the own pages (in the first of them), -]
};
constexpr int kStatePad = 4;
constexpr int kLeastPiece = 32;  // pages

// v of lane 16 (lane / 16) + J
template <int J>
__device__ __forceinline__ float row_lane(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x150 + J, 0xf, 0xf, true));
}
template <int... J, class F>
__device__ __forceinline__ void each(std::integer_sequence<int, J...>, F&& f) {
  (f(std::integral_constant<int, J>{}), ...);
}

__device__ __forceinline__ floatx4 mfma(u32x4 a, u32x4 b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <bool ONCE>
__device__ __forceinline__ u32x4 ld16_kv(const void* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  else return ld16(p);
}

// The lane's number, not kept from before: over a loop it would take a register that the loop needs.
__device__ __forceinline__ int lane_anew() {
  int zero = 0;
  asm volatile("" : "+v"(zero));
  return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
}

// One workgroup's share: a group's pages [lo, hi) of a key/value head, for some of the group's columns.
struct TileWork {
  int kv, row0, c0, cols, state, len, lo, hi;
  int pieces;  // in the first of those that were cut by what there is; else 0
  bool whole;  // there is nothing else of the row and head: the result is written, no state
  int step;  // narrow: pages from one chunk of a wave to its next
  const int32_t* bt;
};

// The r-th longest (by pages, then by number) of up to 64 sequences, one a lane (pages < 0: none): a lane's number.
__device__ __forceinline__ int ranked(int pages, int r, int bits) {
  uint64_t left = __builtin_amdgcn_ballot_w64(pages >= 0);
  for (int b = bits - 1; b >= 0; --b) {
    const uint64_t with = __builtin_amdgcn_ballot_w64((pages >> b) & 1) & left;
    const int n = __builtin_popcountll(with);
    if (r < n) left = with;
    else {
      r -= n;
      left &= ~with;
    }
  }
  const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(left >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)left, 0));
  const int lane = threadIdx.x & 63;
  return __builtin_ctzll(__builtin_amdgcn_ballot_w64(((left >> lane) & 1) && before == r));
}

// Running softmax over N score tiles (scaled by log2 e, -inf where there is no key, or one below fp32's range): p in place of s.
template <int N, int DB>
__device__ __forceinline__ void online_softmax(floatx4 (&s)[N], floatx4 (&acc)[DB], float& m_run, float& l_run) {
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) top = fmaxf(top, s[i][r]);
  top = across_groups<16>(top, MaxOp());
  if (__builtin_amdgcn_ballot_w64(top > m_run) != 0) {  // (rare from the first few tiles on)
    const float m_new = fmaxf(m_run, top);
    const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
    l_run *= alpha;
    m_run = m_new;
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] *= alpha;
  }
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[i][r] = __builtin_amdgcn_exp2f(s[i][r] - m_run);
      sum += s[i][r];
    }
  l_run += sum;
}
struct Probabilities {  // operand B of two tiles
  u32x4 near, rest;
};
__device__ __forceinline__ Probabilities probabilities(const floatx4* s) {
  Probabilities p;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float a = s[w / 2][2 * (w % 2)], b = s[w / 2][2 * (w % 2) + 1];
    p.near[w] = pack_bf16(a, b);
    p.rest[w] = pack_bf16(a - bf16_lo(p.near[w]), b - bf16_hi(p.near[w]));
  }
  return p;
}
template <int T>
__device__ __forceinline__ u32x4 values8(uint32_t a, uint32_t b) {
  const u32x2 lo = values4<T>(a), hi = values4<T>(b);
  return u32x4{lo[0], lo[1], hi[0], hi[1]};
}

// V of bf16 in LDS as it lies in the page: rows 8 banks apart (mod 64) and 16 elements longer than a row, so that the
// transposing reads of half a wave (4 rows of 32 bytes for each of two lane groups, 4 rows apart) meet in no bank.
template <int HD>
constexpr int kVRow = HD + 16;
// Operand A of the second product out of it: lane i of a group of 16 hands in 4 features of key i / 4 and is handed the 4
// keys of feature i; keys 4 g .. 4 g + 3 of two pages.
template <int HD>
__device__ __forceinline__ u32x4 turned(const uint16_t* vfrag, int db) {
  typedef short short4v __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) short4v* lds_short4_ptr;
  const u32x2 p0 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_ptr)(vfrag + 16 * db)));
  const u32x2 p1 = __builtin_bit_cast(
      u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_ptr)(vfrag + kKvPage * kVRow<HD> + 16 * db)));
  return u32x4{p0[0], p0[1], p1[0], p1[1]};
}

// bytes of LDS: a tile of K and of V (wide); the staging areas of the waves (narrow, bf16); the merge (narrow)
template <int HD, int T, bool WIDE>
struct TileLds {
  static constexpr int kK = kWideKeys * HD * 2, kV = kWideKeys * (T == kKvBf16 ? kVRow<HD> : HD) * 2;
  static constexpr int kTile = kK + kV + (T == kKvBf16 ? 0 : 2 * kWideKeys * 4);
  static constexpr int kStage = T == kKvBf16 ? 32 * kVRow<HD> * 2 : 0;
  static constexpr int kMerge = kTileWaves * 16 * (HD + kStatePad) * 4;
  static constexpr int most(int a, int b) { return a > b ? a : b; }
  static constexpr int kBytes = most(WIDE ? kTile : 0, most(kTileWaves * kStage, kMerge));
};

// ---- narrow ----
// 8 bits: of a chunk's 32 keys lane group g has keys 8 (g & 1) .. + 8 of page g / 2: row i of score tile t is key
// 8 (i / 4 & 1) + 4 t + i % 4 of page i / 8.  V is kept with a feature's 16 tokens together: a 16-byte load and two row
// swaps give 8 keys of two blocks of features, operand A as it is wanted.
//   K is asked for one chunk ahead when this one's scores are made, V when its output is: 16 registers each.  (A chunk of 64
// keys has twice those and half the waves: 40 heads, 64 sequences of 545 tokens 76 us, of 32 keys 71.)  Loads that no cache
// keeps: 71 -> 66 there, but one sequence of 700 tokens, which the caches do keep from step to step, 8.6 -> 10.8: kOnceBytes.
template <int HD, int T, bool ONCE>
__device__ __forceinline__ void narrow_quant(const TileArgs& a, const TileWork& w, const u32x4 (&qf)[HD / 32],
                                             floatx4 (&acc)[HD / 16], float& m_run, float& l_run) {
  constexpr int KL = HD / 64, VL = HD / 32;  // 16-byte loads of a key, of a chunk's V, per lane
  const int lane = threadIdx.x & 63, hl = lane & 15, g = lane >> 4;
  const uint8_t* kc = static_cast<const uint8_t*>(a.k);
  const uint8_t* vc = static_cast<const uint8_t*>(a.v);
  int kid = 0, vid = 0;
  auto ids = [&](int p) {  // pages of the lane as a row of K and as a column of V (behind the last: the last, without keys)
    kid = w.bt[min(p + (hl >> 3), w.hi - 1)];
    vid = w.bt[min(p + (g >> 1), w.hi - 1)];
  };
  u32x4 kr[2][KL], vr[VL];
  uint16_t ksr, vsr;
  const uint8_t* vsrc;
  auto fetch_k = [&] {
    const size_t kp = (size_t)kid * a.n_kv_heads + w.kv, vp = (size_t)vid * a.n_kv_heads + w.kv;
    const uint8_t* src = kc + kp * (kKvPage * HD) + (8 * ((hl >> 2) & 1) + (hl & 3)) * HD + 16 * g;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < KL; ++c) kr[t][c] = ld16_kv<ONCE>(src + 4 * t * HD + 64 * c);
    const size_t sc = vp * kKvPage + 8 * (g & 1) + (hl & 7);
    ksr = a.k_scale[sc];
    vsr = a.v_scale[sc];
    vsrc = vc + vp * (kKvPage * HD) + (16 * (g & 1) + hl) * kKvPage;
  };
  auto fetch_v = [&] {
#pragma unroll
    for (int i = 0; i < VL; ++i) vr[i] = ld16_kv<ONCE>(vsrc + 32 * i * kKvPage);
  };
  int pg = w.lo;
  if (pg < w.hi) {
    ids(pg);
    fetch_k();
    fetch_v();
    ids(pg + w.step);
  }
  for (; pg < w.hi; pg += w.step) {
    // keys of the lane's half page
    const int there = pg + (g >> 1) < w.hi ? min(w.len - (pg + (g >> 1)) * kKvPage - 8 * (g & 1), 8) : 0;
    floatx4 s[2] = {floatx4{0.f, 0.f, 0.f, 0.f}, floatx4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int c = 0; c < KL; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          s[t] = mfma(values8<T>(kr[t][c][2 * h], kr[t][c][2 * h + 1]), qf[2 * c + h], s[t]);
    const float ks = bf16_lo(ksr) * a.scale_log2e, vs = (hl & 7) < there ? bf16_lo(vsr) : 0.f;
    const bool more = pg + w.step < w.hi;
    if (more) fetch_k();
    each(std::make_integer_sequence<int, 8>{}, [&](auto j) {
      const float x = s[j() / 4][j() % 4] * row_lane<j()>(ks);
      s[j() / 4][j() % 4] = j() < there ? x : -INFINITY;  // (whatever the slot holds)
    });
    online_softmax(s, acc, m_run, l_run);
    each(std::make_integer_sequence<int, 8>{}, [&](auto j) { s[j() / 4][j() % 4] *= row_lane<j()>(vs); });
    const Probabilities pf = probabilities(s);
    // A load gave the lane 16 keys of one feature, g & 1 choosing between two blocks of 16 features: words 2, 3 of the
    // even rows of lanes against words 0, 1 of the odd ones, and words 0, 1 are 8 keys of the first block in every lane,
    // words 2, 3 of the second.
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      uint32_t x[4] = {vr[i][0], vr[i][1], vr[i][2], vr[i][3]};
      swap16(x[0], x[2]);
      swap16(x[1], x[3]);
      vr[i] = u32x4{x[0], x[1], x[2], x[3]};
    }
    // slots behind the end may hold NaN, and 0 * NaN is NaN
    if (__builtin_amdgcn_ballot_w64(there < 8) != 0) {
      const uint32_t keep0 = there >= 4 ? 0xffffffffu : (1u << (8 * max(there, 0))) - 1u;
      const uint32_t keep1 = there >= 8 ? 0xffffffffu : (1u << (8 * max(there - 4, 0))) - 1u;
#pragma unroll
      for (int i = 0; i < VL; ++i) vr[i] &= u32x4{keep0, keep1, keep0, keep1};
    }
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const u32x4 v[2] = {values8<T>(vr[i][0], vr[i][1]), values8<T>(vr[i][2], vr[i][3])};
#pragma unroll
      for (int h = 0; h < 2; ++h) acc[2 * i + h] = mfma(v[h], pf.near, acc[2 * i + h]);
#pragma unroll
      for (int h = 0; h < 2; ++h) acc[2 * i + h] = mfma(v[h], pf.rest, acc[2 * i + h]);
    }
    if (more) {
      fetch_v();
      ids(pg + 2 * w.step);
    }
  }
}

// bf16: row i of score tile t is key i of page t; V goes through the wave's own LDS.
template <int HD, bool ONCE>
__device__ __forceinline__ void narrow_bf16(const TileArgs& a, const TileWork& w, const u32x4 (&qf)[HD / 32],
                                            floatx4 (&acc)[HD / 16], float& m_run, float& l_run, unsigned char* smem) {
  constexpr int CPR = HD / 8, RPL = 64 / CPR;  // 16-byte pieces of a row, rows of a load
  constexpr int NL = kKvPage / RPL;            // loads of a page
  const int lane = threadIdx.x & 63, hl = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint16_t* kc = static_cast<const uint16_t*>(a.k);
  const uint16_t* vc = static_cast<const uint16_t*>(a.v);
  uint16_t* vst = reinterpret_cast<uint16_t*>(smem) + wave * 32 * kVRow<HD>;
  const int vrow = lane / CPR, vcol = lane % CPR * 8;
  int id[2] = {0, 0};
  auto ids = [&](int p) {
#pragma unroll
    for (int u = 0; u < 2; ++u) id[u] = w.bt[min(p + u, w.hi - 1)];
  };
  u32x4 kr[2][HD / 32], vr[2][NL];
  size_t at[2];
  auto fetch_k = [&] {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      at[u] = ((size_t)id[u] * a.n_kv_heads + w.kv) * (kKvPage * HD);
#pragma unroll
      for (int s = 0; s < HD / 32; ++s) kr[u][s] = ld16_kv<ONCE>(kc + at[u] + hl * HD + 32 * s + 8 * g);
    }
  };
  auto fetch_v = [&] {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < NL; ++i) vr[u][i] = ld16_kv<ONCE>(vc + at[u] + (size_t)(RPL * i + vrow) * HD + vcol);
  };
  int pg = w.lo;
  if (pg < w.hi) {
    ids(pg);
    fetch_k();
    fetch_v();
    ids(pg + w.step);
  }
  for (; pg < w.hi; pg += w.step) {
    int there[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) there[u] = pg + u < w.hi ? min(w.len - (pg + u) * kKvPage, kKvPage) : 0;
    floatx4 s[2] = {floatx4{0.f, 0.f, 0.f, 0.f}, floatx4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int st = 0; st < HD / 32; ++st)
#pragma unroll
      for (int u = 0; u < 2; ++u) s[u] = mfma(kr[u][st], qf[st], s[u]);
    const bool more = pg + w.step < w.hi;
    if (more) fetch_k();
    // (rows behind the end as zeros: what is there may be NaN, and 0 * NaN is NaN)
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int row = RPL * i + vrow;
        *reinterpret_cast<u32x4*>(vst + (u * kKvPage + row) * kVRow<HD> + vcol) =
            row < there[u] ? vr[u][i] : u32x4{0, 0, 0, 0};
      }
    if (more) {
      fetch_v();
      ids(pg + 2 * w.step);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[u][r] = 4 * g + r < there[u] ? s[u][r] * a.scale_log2e : -INFINITY;
    online_softmax(s, acc, m_run, l_run);
    const Probabilities pf = probabilities(s);
    __builtin_amdgcn_wave_barrier();  // (a wave's LDS accesses keep their order; the compiler has to keep it too)
    const uint16_t* vfrag = vst + (4 * g + (hl >> 2)) * kVRow<HD> + (hl & 3) * 4;
#pragma unroll
    for (int db = 0; db < HD / 16; db += 2) {
      const u32x4 v[2] = {turned<HD>(vfrag, db), turned<HD>(vfrag, db + 1)};
#pragma unroll
      for (int h = 0; h < 2; ++h) acc[db + h] = mfma(v[h], pf.near, acc[db + h]);
#pragma unroll
      for (int h = 0; h < 2; ++h) acc[db + h] = mfma(v[h], pf.rest, acc[db + h]);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// ---- wide ----
// A tile is 64 keys, in two halves.  K in LDS as bf16 rows, chunk c of 16 bytes at c ^ swizzle: the 16 rows that an operand
// read takes at one chunk number then lie in 16 different places of the 256 bytes of all banks.  bf16: row i of score tile t
// of a half is its key 16 t + i, and V is as for the narrow form.  8 bits: row i is key 8 (i / 4) + 4 t + i % 4, so that lane
// group g has keys 8 g .. + 8, and V^T rows of 64 keys hold operand A of half u in their chunk 4 u + g (swizzled by d / 2).
//   The next tile's bytes are in registers while this one is multiplied.  (Tiles of 32 keys in two buffers, one barrier each:
// the same LDS and barriers, but twice the chains of dependent steps per key; 40 rows of 64 heads on 8 behind 6951 tokens,
// unsplit, 167 us instead of 141.)  A tile takes a lone workgroup 1.2 us, and three on a compute unit 2.5 together: 280 vector
// instructions a wave and tile, a third of them staging, beside 32 products.  32 x 32 x 16 instructions with half the operand
// reads (each wave 32 columns over half of the keys), operands asked for all together, and K's scale with the conversion were
// no faster.
template <int HD, int T>
__device__ __forceinline__ int k_swizzle(int row) {
  if constexpr (T == kKvBf16) return HD == 128 ? row & 15 : (row >> 1) & 7;
  else return HD == 128 ? (row & 3) | ((row >> 3) & 3) << 2 : ((row >> 1) & 1) | ((row >> 3) & 3) << 1;
}

template <int HD, int T>
__device__ __forceinline__ void wide_tiles(const TileArgs& a, const TileWork& w, const u32x4 (&qf)[HD / 32],
                                           floatx4 (&acc)[HD / 16], float& m_run, float& l_run, bool idle,
                                           unsigned char* smem) {
  using L = TileLds<HD, T, true>;
  constexpr bool kQuant = T != kKvBf16;
  constexpr int B8 = HD / 8;                     // numbers of a page's K, and of its V, in a thread: 16 or 8
  constexpr int RW = kQuant ? B8 / 4 : B8 / 2;   // words of them
  constexpr int NCH = B8 / 8;                    // 16-byte chunks of bf16
  constexpr int kPages = kWideKeys / kKvPage;
  const int tid = threadIdx.x, lane = tid & 63, hl = lane & 15, g = lane >> 4;
  // the thread's pages are those 2 u + odd of a tile, in each of them the same place
  const int odd = __builtin_amdgcn_readfirstlane(tid >> 7), at = tid & 127;
  const int key = at >> 3, piece = at & 7;       // of K (and of V where it is bf16): B8 numbers from B8 piece on
  uint16_t* kt = reinterpret_cast<uint16_t*>(smem);
  uint16_t* vt = reinterpret_cast<uint16_t*>(smem + L::kK);
  float* sc = reinterpret_cast<float*>(smem + L::kK + L::kV);  // scales of K, of V
  uint32_t kr[2][RW], vr[2][RW];
  uint16_t scale[2] = {0, 0};
  int id[2] = {0, 0}, pg;
  auto ids = [&](int p) {
#pragma unroll
    for (int u = 0; u < 2; ++u) id[u] = w.bt[min(p + 2 * u + odd, w.hi - 1)];
  };
  auto words = [&](uint32_t (&r)[RW], const void* p) {
    if constexpr (RW == 2) {
      const u32x2 x = *static_cast<const u32x2*>(p);
      r[0] = x[0];
      r[1] = x[1];
    } else {
#pragma unroll
      for (int i = 0; i < RW; i += 4) {
        const u32x4 x = ld16(static_cast<const char*>(p) + 4 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) r[i + j] = x[j];
      }
    }
  };
  auto fetch = [&] {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const size_t page = (size_t)id[u] * a.n_kv_heads + w.kv;
      const size_t first = page * (kKvPage * HD) + (size_t)at * B8;
      if constexpr (kQuant) {
        words(kr[u], static_cast<const uint8_t*>(a.k) + first);
        words(vr[u], static_cast<const uint8_t*>(a.v) + first);
        if (at < 32) scale[u] = (at < 16 ? a.k_scale : a.v_scale)[page * kKvPage + (at & 15)];
      } else {
        words(kr[u], static_cast<const uint16_t*>(a.k) + first);
        words(vr[u], static_cast<const uint16_t*>(a.v) + first);
      }
    }
  };
  auto stage = [&] {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int page = 2 * u + odd, row = page * kKvPage + key;
      const int there = pg + page < w.hi ? min(w.len - (pg + page) * kKvPage, kKvPage) : 0;  // keys of the page
      if constexpr (kQuant) {
#pragma unroll
        for (int c = 0; c < NCH; ++c)
          *reinterpret_cast<u32x4*>(kt + row * HD + ((NCH * piece + c) ^ k_swizzle<HD, T>(row)) * 8) =
              values8<T>(kr[u][2 * c], kr[u][2 * c + 1]);
        // the thread's V: feature `at` of the page, all tokens (HD 128), or feature at / 2, half of them
        const int d = HD == 128 ? at : at >> 1, t0 = HD == 128 ? 0 : 8 * (at & 1);
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
          uint32_t x = vr[u][2 * c], y = vr[u][2 * c + 1];
          if (there < kKvPage) {  // slots behind the end may hold NaN
            const int n = there - t0 - 8 * c;
            x = n >= 4 ? x : n > 0 ? x & ((1u << (8 * n)) - 1u) : 0;
            y = n >= 8 ? y : n > 4 ? y & ((1u << (8 * (n - 4))) - 1u) : 0;
          }
          *reinterpret_cast<u32x4*>(vt + d * kWideKeys + ((2 * page + t0 / 8 + c) ^ ((d >> 1) & 7)) * 8) = values8<T>(x, y);
        }
        if (at < 32) {
          const float f = bf16_lo(scale[u]);
          sc[(at < 16 ? 0 : kWideKeys) + page * kKvPage + (at & 15)] =
              at < 16 ? f * a.scale_log2e : ((at & 15) < there ? f : 0.f);
        }
      } else {
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
          *reinterpret_cast<u32x4*>(kt + row * HD + ((NCH * piece + c) ^ k_swizzle<HD, T>(row)) * 8) =
              u32x4{kr[u][4 * c], kr[u][4 * c + 1], kr[u][4 * c + 2], kr[u][4 * c + 3]};
          *reinterpret_cast<u32x4*>(vt + row * kVRow<HD> + (NCH * piece + c) * 8) =
              key < there ? u32x4{vr[u][4 * c], vr[u][4 * c + 1], vr[u][4 * c + 2], vr[u][4 * c + 3]} : u32x4{0, 0, 0, 0};
        }
      }
    }
  };
  pg = w.lo;
  if (pg >= w.hi) return;
  ids(pg);
  fetch();
  ids(pg + kPages);
  for (; pg < w.hi; pg += kPages) {
    if (pg != w.lo) lds_barrier();  // every wave is done with the last tile
    stage();
    if (pg + kPages < w.hi) {
      fetch();
      ids(pg + 2 * kPages);
    }
    lds_barrier();
    if (idle) continue;
    floatx4 s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < HD / 32; ++st)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int row = 32 * (t / 2) + (kQuant ? 8 * (hl >> 2) + 4 * (t % 2) + (hl & 3) : 16 * (t % 2) + hl);
        s[t] = mfma(ld16(kt + row * HD + ((4 * st + g) ^ k_swizzle<HD, T>(row)) * 8), qf[st], s[t]);
      }
    // keys from this tile on, of the sequence and of this split
    const int here = min(w.len - pg * kKvPage, (w.hi - pg) * kKvPage);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if constexpr (kQuant) s[t] *= *reinterpret_cast<const floatx4*>(sc + 32 * (t / 2) + 8 * g + 4 * (t % 2));
      else s[t] *= a.scale_log2e;
    }
    if (here < kWideKeys) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (32 * (t / 2) + (kQuant ? 8 * g + 4 * (t % 2) : 16 * (t % 2) + 4 * g) + r >= here) s[t][r] = -INFINITY;
    }
    online_softmax(s, acc, m_run, l_run);
    if constexpr (kQuant) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
        s[t] *= *reinterpret_cast<const floatx4*>(sc + kWideKeys + 32 * (t / 2) + 8 * g + 4 * (t % 2));
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const Probabilities pf = probabilities(s + 2 * u);
#pragma unroll
      for (int db = 0; db < HD / 16; ++db) {
        if constexpr (kQuant) {
          const int d = 16 * db + hl;
          acc[db] = mfma(ld16(vt + d * kWideKeys + ((4 * u + g) ^ ((d >> 1) & 7)) * 8), pf.near, acc[db]);
        } else {
          const u32x4 v = turned<HD>(vt + (32 * u + 4 * g + (hl >> 2)) * kVRow<HD> + (hl & 3) * 4, db);
          acc[db] = mfma(v, pf.rest, mfma(v, pf.near, acc[db]));
        }
      }
    }
  }
}

// What a wave has of a lane's column that is all there is of it in this split: a state, or the result.
template <int HD>
__device__ __forceinline__ void store_columns(const TileArgs& a, const TileWork& w, int col, const floatx4 (&acc)[HD / 16],
                                              float m, float l) {
  if (col >= w.cols) return;
  const int g = lane_anew() >> 4, G = a.n_heads / a.n_kv_heads;
  const size_t item = (size_t)(w.row0 + col / G) * a.n_heads + w.kv * G + col % G;
  float* st = a.partial + (item * a.n_states + w.state) * (HD + kStatePad);
  if (w.pieces > 0 && g == 0) reinterpret_cast<int*>(st)[HD + 2] = w.pieces;
  if (w.whole) {
    const float inv = l == 0.f ? 0.f : 1.f / l;  // no key at all: 0
#pragma unroll
    for (int db = 0; db < HD / 16; ++db)
      *reinterpret_cast<u32x2*>(a.o + item * HD + 16 * db + 4 * g) =
          u32x2{pack_bf16(acc[db][0] * inv, acc[db][1] * inv), pack_bf16(acc[db][2] * inv, acc[db][3] * inv)};
  } else {
#pragma unroll
    for (int db = 0; db < HD / 16; ++db) *reinterpret_cast<floatx4*>(st + 16 * db + 4 * g) = acc[db];
    if (g == 0) {
      st[HD] = m;
      st[HD + 1] = l;
    }
  }
}

// WIDE: either part may be wide (a part of up to 16 columns is narrow all the same).  ONCE: the rows' own pages are read
// with loads that no cache keeps.  JOINED: part 0 has no workgroups, a row's take its group's prefix and then its own pages.
template <int HD, int T, bool WIDE, bool ONCE, bool JOINED>
__global__ __launch_bounds__(kTileThreads) __attribute__((amdgpu_waves_per_eu(WIDE || (JOINED && T == kKvBf16) ? 3 : 4))) void tile_attention_kernel(
    const TileArgs a) {
  constexpr int DB = HD / 16, kSteps = HD / 32, kState = HD + kStatePad;
  constexpr bool kQuant = T != kKvBf16;
  __shared__ __attribute__((aligned(16))) unsigned char smem[TileLds<HD, T, WIDE>::kBytes];
  const int tid = threadIdx.x, lane = tid & 63, hl = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool second = (int)blockIdx.x >= a.first_blocks;
  const TilePart& p = a.part[second ? 1 : 0];
  const bool wide = WIDE && p.wide;
  const int G = a.n_heads / a.n_kv_heads;

  // workgroup -> key/value head (fastest), block of columns, group, split.  (With the splits of a sequence next to each other
  // those without pages come in between, and what has some is dealt to the same few compute units: three times as long.)
  int id = (int)blockIdx.x - (second ? a.first_blocks : 0);
  const int x = id % p.blocks_x;
  id /= p.blocks_x;
  int group = id % p.groups;
  const int split = id / p.groups;
  TileWork w;
  w.kv = p.solo ? kTileWaves * x + wave : x % a.n_kv_heads;
  if (w.kv >= a.n_kv_heads) return;
  // Workgroups reach the chip's eight partitions in turn: heads that share 128 bytes of scales meet in one of them.
  if (kQuant && !p.solo && a.n_kv_heads % 8 == 0) w.kv = w.kv % 8 * (a.n_kv_heads / 8) + w.kv / 8;
  w.c0 = wide ? x / a.n_kv_heads * kWideCols : 0;
  if (p.rank) {
    // Longest first among every n-th sequence, so that no long one starts among the last and ends the launch by itself.
    const int n = (p.groups + 63) / 64, other = group % n + n * lane;
    const int len = other < p.groups ? max(p.lens[other] + p.len_add, 0) : -2 * kKvPage;
    const int at = ranked(min((len + kKvPage - 1) / kKvPage, p.max_pages), group / n, 32 - __builtin_clz(p.max_pages));
    group = group % n + n * at;
    w.len = __builtin_amdgcn_readlane(len, at);
  } else {
    w.len = p.lens[group] + p.len_add;
  }
  w.len = min(w.len, p.max_len);
  w.row0 = p.cu_rows ? p.cu_rows[group] : group;
  w.cols = (p.cu_rows ? p.cu_rows[group + 1] - w.row0 : 1) * G;
  if (w.c0 >= w.cols) return;
  const int pages = (w.len + kKvPage - 1) / kKvPage;
  int piece = p.pages_per_split;
  w.pieces = 0;
  w.whole = a.n_states == 1;
  if (piece == 0) {
    // A piece is two thirds of what each compute unit has of all pages: equal sequences stay whole where they are enough
    // for the chip, and those are cut that would end the launch by themselves.  What is whole needs no state.
    float all = 0.f;
    for (int i0 = 0; i0 < p.groups; i0 += 64) {
      const int i = i0 + lane;
      if (i < p.groups) all += (float)((max(min(p.lens[i] + p.len_add, p.max_len), 0) + kKvPage - 1) / kKvPage);
    }
    const int fair = (int)fminf(wave_sum(all) * (float)p.blocks_x * (1.f / 384.f), 1e9f);
    const int most = __builtin_amdgcn_readfirstlane(max(fair, kLeastPiece));
    const int cuts = min((pages + most - 1) / most, p.splits);
    piece = cuts <= 1 ? max(pages, 1) : ((pages + cuts - 1) / cuts + 7) & ~7;  // (8: a chunk for each wave)
    const int pieces = max((pages + piece - 1) / piece, 1);
    if (split >= pieces) return;
    if (split == 0) w.pieces = pieces;
    w.whole = pieces == 1 && p.first_state == 0;
  }
  w.lo = split * piece;
  w.hi = min(pages, w.lo + piece);
  w.bt = p.tables + (size_t)group * p.max_pages;
  w.state = p.first_state + split;
  w.step = p.solo ? 2 : 2 * kTileWaves;
  if (!wide && !p.solo) w.lo += 2 * wave;

  // Operand B of the scores.  8 bits, narrow: instruction 2 c + h takes features 64 c + 16 g + 8 h .. + 8 of lane group g (16
  // bytes of K are two operands); else instruction s features 32 s + 8 g .. + 8.
  const int my_c0 = w.c0 + (wide ? 16 * wave : 0), col = my_c0 + hl;
  u32x4 qf[kSteps];
  {
    const uint16_t* qp = a.q + (size_t)(w.row0 + col / G) * a.q_stride + (size_t)(w.kv * G + col % G) * HD;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      qf[s] = u32x4{0, 0, 0, 0};
      const int at = kQuant && !wide ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
      if (col < w.cols) qf[s] = ld16(qp + at);
    }
  }
  floatx4 acc[DB];
  float m_run = kLowestScore, l_run = 0.f;  // l_run: this lane's share of the sum
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = floatx4{0.f, 0.f, 0.f, 0.f};

  if constexpr (WIDE) {
    if (wide) {
      wide_tiles<HD, T>(a, w, qf, acc, m_run, l_run, my_c0 >= w.cols, smem);
      return store_columns<HD>(a, w, col, acc, m_run, across_groups<16>(l_run, AddOp()));
    }
  }
  TileWork next;
  if constexpr (JOINED) {
    const TilePart& pre = a.part[0];
    int of = 0;  // the row's group: as many end at the row or before
    for (int i0 = 0; i0 < pre.groups; i0 += 64)
      of += __builtin_popcountll(
          __builtin_amdgcn_ballot_w64(i0 + lane < pre.groups && pre.cu_rows[min(i0 + lane, pre.groups - 1) + 1] <= group));
    of = min(of, pre.groups - 1);
    next = w;
    w.len = min(pre.lens[of], pre.max_len);
    w.hi = (w.len + kKvPage - 1) / kKvPage;
    w.bt = pre.tables + (size_t)of * pre.max_pages;
    if (!p.solo) next.lo = 2 * ((wave - (w.hi + 1) / 2) & (kTileWaves - 1));  // (the wave whose turn it is)
  }
#pragma unroll 1
  for (int seg = JOINED ? 0 : 1; seg < 2; ++seg) {
    if constexpr (kQuant) narrow_quant<HD, T, ONCE>(a, w, qf, acc, m_run, l_run);
    else narrow_bf16<HD, ONCE>(a, w, qf, acc, m_run, l_run, smem);
    if constexpr (JOINED) w = next;
  }
  if (p.solo) return store_columns<HD>(a, w, lane_anew() & 15, acc, m_run, across_groups<16>(l_run, AddOp()));

  // Merge the waves.  A wave without keys has the lowest maximum and sum and output 0.  (Where scores are NaN, so is the sum.)
  const int thread = 64 * wave + lane_anew();
  const float l = across_groups<16>(l_run, AddOp());
  float* mg = reinterpret_cast<float*>(smem);  // [wave][column][output[HD], max, sum, -, -]
  __syncthreads();                             // the staging areas are done with
  float* dst = mg + (thread >> 6 << 4 | (thread & 15)) * kState;
  const int mg_g = thread >> 4 & 3;
#pragma unroll
  for (int db = 0; db < DB; ++db) *reinterpret_cast<floatx4*>(dst + 16 * db + 4 * mg_g) = acc[db];
  if (mg_g == 0) {
    dst[HD] = m_run;
    dst[HD + 1] = l;
  }
  __syncthreads();
  constexpr int ND = HD / 16;
  const int c = thread >> 4, d0 = (thread & 15) * ND;
  if (c >= w.cols) return;
  float m = kLowestScore, sum = 0.f, out[ND];
#pragma unroll
  for (int i = 0; i < kTileWaves; ++i) m = fmaxf(m, mg[(i * 16 + c) * kState + HD]);
#pragma unroll
  for (int j = 0; j < ND; ++j) out[j] = 0.f;
#pragma unroll
  for (int i = 0; i < kTileWaves; ++i) {
    const float* src = mg + (i * 16 + c) * kState;
    const float f = __builtin_amdgcn_exp2f(src[HD] - m);
    sum += src[HD + 1] * f;
#pragma unroll
    for (int j = 0; j < ND; ++j) out[j] += src[d0 + j] * f;
  }
  const size_t to = (size_t)(w.row0 + c / G) * a.n_heads + w.kv * G + c % G;
  float* st = a.partial + (to * a.n_states + w.state) * kState;
  if (w.pieces > 0 && (thread & 15) == 0) reinterpret_cast<int*>(st)[HD + 2] = w.pieces;
  if (w.whole) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;  // no key at all: 0
    uint32_t v[ND / 2];
#pragma unroll
    for (int j = 0; j < ND / 2; ++j) v[j] = pack_bf16(out[2 * j] * inv, out[2 * j + 1] * inv);
    uint16_t* op = a.o + to * HD + d0;
    if constexpr (ND == 8) st16(op, u32x4{v[0], v[1], v[2], v[3]});
    else *reinterpret_cast<u32x2*>(op) = u32x2{v[0], v[1]};
  } else {
#pragma unroll
    for (int j = 0; j < ND; j += 4) *reinterpret_cast<floatx4*>(st + d0 + j) = floatx4{out[j], out[j + 1], out[j + 2], out[j + 3]};
    if ((thread & 15) == 0) {
      st[HD] = m;
      st[HD + 1] = sum;
    }
  }
}

// The states of a (row, head) as one, in a fixed order: the same bits whenever.  counted >= 0: behind that many there are as
// many as the next one says.  W waves take a (row, head), wave w states w,
// w + W, ...: its lanes have the maxima and sums of 64 of them at once, and then HD / 64 features each, the states asked for 8
// at a time.
template <int HD, int W>
__global__ __launch_bounds__(kTileThreads) void tile_combine_kernel(const float* __restrict__ partial, int items, int stride,
                                                                    int counted, uint16_t* __restrict__ o) {
  constexpr int ND = HD / 64, kState = HD + kStatePad, U = 8;
  __shared__ float merge[W == 1 ? 1 : W][HD + 2];
  const int lane = threadIdx.x & 63, in_wg = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = in_wg % W;
  const size_t item = (size_t)blockIdx.x * (kTileWaves / W) + in_wg / W;
  if (item >= (size_t)items) return;  // (W = 1: a wave by itself; else never)
  const float* src = partial + item * stride * kState;
  int n_states = stride;
  if (counted >= 0) {  // (one in all: the result is there already)
    n_states = counted + __builtin_amdgcn_readfirstlane(reinterpret_cast<const int*>(src)[counted * kState + HD + 2]);
    if (n_states <= 1) return;
  }
  float m_run = kLowestScore, l_run = 0.f, out[ND] = {};
  for (int s0 = wave; s0 < n_states; s0 += 64 * W) {
    const int n = min((n_states - s0 + W - 1) / W, 64);  // of them in this turn
    float m = kLowestScore, l = 0.f;
    if (lane < n) {
      m = src[(size_t)(s0 + W * lane) * kState + HD];
      l = src[(size_t)(s0 + W * lane) * kState + HD + 1];
    }
    float v[U][ND];
    auto load = [&](int i0) {  // (behind the last: the last again, not used)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float* st = src + (size_t)(s0 + W * min(i0 + u, n - 1)) * kState + ND * lane;
#pragma unroll
        for (int j = 0; j < ND; ++j) v[u][j] = st[j];
      }
    };
    load(0);
    float top = lane_op<1>(m, MaxOp());
    top = lane_op<2>(top, MaxOp());
    top = lane_op<kMirror4>(top, MaxOp());
    top = across_groups<8>(top, MaxOp());
    const float m_new = fmaxf(m_run, top), alpha = __builtin_amdgcn_exp2f(m_run - m_new);
    const float f = __builtin_amdgcn_exp2f(m - m_new);
    l_run = l_run * alpha + wave_sum(l * f);
#pragma unroll
    for (int j = 0; j < ND; ++j) out[j] *= alpha;
    m_run = m_new;
    for (int i0 = 0; i0 < n; i0 += U) {
      if (i0 > 0) load(i0);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float fu = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), min(i0 + u, n - 1)));
        if (i0 + u < n)
#pragma unroll
          for (int j = 0; j < ND; ++j) out[j] += v[u][j] * fu;
      }
    }
  }
  if constexpr (W == 1) {
    const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
    if constexpr (ND == 2) reinterpret_cast<uint32_t*>(o)[item * 64 + lane] = pack_bf16(out[0] * inv, out[1] * inv);
    else reinterpret_cast<__bf16*>(o)[item * HD + lane] = (__bf16)(out[0] * inv);
    return;
  }
#pragma unroll
  for (int j = 0; j < ND; ++j) merge[wave][ND * lane + j] = out[j];
  if (lane == 0) {
    merge[wave][HD] = m_run;
    merge[wave][HD + 1] = l_run;
  }
  __syncthreads();
  const int d = threadIdx.x;
  if (d >= HD) return;
  float m = kLowestScore, sum = 0.f, r = 0.f;
#pragma unroll
  for (int i = 0; i < W; ++i) m = fmaxf(m, merge[i][HD]);
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const float f = __builtin_amdgcn_exp2f(merge[i][HD] - m);
    sum += merge[i][HD + 1] * f;
    r += merge[i][d] * f;
  }
  reinterpret_cast<__bf16*>(o)[item * HD + d] = (__bf16)(sum == 0.f ? 0.f : r / sum);
}

// ---- plans ----
constexpr double kOnceBytes = 256e6;  // of own pages: more than the last-level cache could keep until the next step

// A key/value head for each wave (`items` of them over all rows) instead of four waves for each: nothing to merge, four times as
// many at once, but a sequence takes as long as one wave needs.  Of 40 heads (us, four waves and one): 64 sequences of 10
// tokens 12.3 and 6.8, of 60 14.7 and 11.4, of 260 43.7 and 40.7, of 545 65.9 and 71.4; 16 of 130 9.3 and 9.0, 8 of 130 7.6
// and 8.5; 8 key/value heads, 64 of 260 11.4 and 13.0, 128 of 260 17.0 and 15.3.  (256 of 1100 on 8 key/value heads, equal
// ones, take 118 and 99, but 128 ragged ones up to 2048 on 40 heads 105 and 140.)
static bool solo_of(long items, long max_len) {
  return max_len <= 32 || (items >= 320 && max_len <= 64) || (items >= 1024 && max_len <= 320);
}
static int blocks_of(long cols) { return (int)(cols <= kNarrowCols ? 1 : (cols + kWideCols - 1) / kWideCols); }

// Where there are 512 workgroups or more without a split: cut by how unequal the sequences are, which only the launch can see,
// if the longest there may be takes a workgroup (0.2 us a page) clearly longer than such a batch takes at a fifth of the bound,
// and the second launch.  Of 166 batches of 512 to 1088 (lognormal, uniform and equal lengths up to 1024 to 16000 tokens) 2.8 %
// slower than the best of none and 12 ways to cut for each; none cut 9.8 %.  (us, none cut and cut, 64 rows of 64 heads on 8:
// lognormal up to 4096 tokens 55 and 32, up to 2048 32 and 26, up to 1024 17.3 and 19.8; uniform up to 4096 64 and 64; all of
// 4096 88.9 and 91.5.)
static bool cut_of(long items, long max_len) {
  const double pages = (double)((max_len + kKvPage - 1) / kKvPage);
  return items >= 512 && pages * (0.2 - 0.000163 * (double)items) > 12.0;
}

// Splits of up to max_len tokens for `items` workgroups that there are anyway; with cut_of the most there may be.  Where they are
// fewer than two per compute unit and the pages 48 or more: enough for three, of 8 pages (a chunk for each wave) or more, of 48
// where there are 160 workgroups already.  Below that the second launch, which joins them, costs what the splits save.  Of 115
// batches of three layer shapes (4 to 1200 items, 500 to 60000 tokens, equal and ragged) these splits are 4 % slower than the
// best of up to 13 numbers each; 8 pages everywhere 6 %.
static int tile_splits(long items, long max_len) {
  const long pages = (max_len + kKvPage - 1) / kKvPage;
  if (cut_of(items, max_len)) return (int)std::max(2l, std::min(4096 / items, pages / kLeastPiece));
  if (items >= 512 || pages < 48) return 1;
  return (int)std::max(1l, std::min((768 + items - 1) / items, pages / (items < 160 ? 8 : 48)));
}

// Splits of prefixes of up to max_prefix tokens: at most 1.75 workgroups per compute unit, of 6 pages or more, and no more
// than pay: halving a workgroup's share of the pages saves 0.3 us a page, each state of a row and head costs 0.3 ns (1056 bytes
// written and read).  254 calls (2 to 128 rows in 1 or 3 groups, four layer shapes, 100 to 12000 tokens, on e4m3 and bf16): 3.7 %
// slower than the best number for each; 512 workgroups of 8 pages by themselves 5.2 %.
//   Where the rows' own pages keep the chip busy for longer, fewer do: down to a third, since max_len may be a generous bound.
// (40 heads, 64 rows of 16 to 256 bf16 tokens behind 2048: 7 splits 52 us, 2 of them 46.)
static int prefix_splits(int B, int n_heads, int n_kv_heads, int n_groups, int max_prefix, double own_bytes) {
  const long items = (long)n_kv_heads * std::max(n_groups, blocks_of((long)B * (n_heads / n_kv_heads)));
  const int pages = (max_prefix + kKvPage - 1) / kKvPage;
  const double paying = std::min(std::sqrt(900.0 * pages / ((double)B * n_heads)), (double)((448 + items - 1) / items));
  const double own_us = own_bytes / 2 / 5.5e6;  // (half of the bound, at 5.5 TB/s)
  const double enough = std::max(paying / 3, std::min(paying, 0.3 * pages / std::max(own_us, 1e-3)));
  return (int)std::max(1l, std::min((long)(enough + 0.5), (long)pages / 6));
}

// One launch in which every row reads its group's prefix for itself, and no states: where the prefix is short or the rows are
// few.  The bytes read again, out of caches, cost 0.1 us a MB, the states of a row and head 0.25 ns each, the second launch 2.4
// us.  836 calls (1 to 160 rows in 1 or 4 groups, three layer shapes, prefixes of 16 to 800 tokens, own tokens up to 700, all
// types): 0.4 % slower than the better way for each; two parts always 23 %, joined always 11 %.  (us, two parts and joined: 5
// rows of 4 heads behind 45 tokens 7.6 and 5.0; e4m3, 64 rows of 64 heads on 8 behind 200 11.8 and 8.3; 64 rows of 40 heads
// behind 200 11.9 and 21.3.)
static bool joined_of(int splits, int B, int n_heads, int n_kv_heads, int head_dim, int kv_type, int max_len, int max_prefix,
                      double own_bytes) {
  const int G = n_heads / n_kv_heads;
  if (G > kNarrowCols || own_bytes > kOnceBytes) return false;
  if (tile_splits((long)B * n_kv_heads, (long)max_len + max_prefix) > 1) return false;
  const double again = (double)B * max_prefix * n_kv_heads * head_dim * (kv_type == kKvBf16 ? 4 : 2);
  return again * 0.1e-6 < 2.4 + 0.25e-3 * B * n_heads * (splits + 1.0);
}

TilePlan tile_plan(int B, int n_heads, int n_kv_heads, int head_dim, int kv_type, int max_len, int n_groups, int max_prefix) {
  TilePlan p;
  p.own = tile_splits((long)B * n_kv_heads * blocks_of(n_heads / n_kv_heads), max_len);
  p.cut = cut_of((long)B * n_kv_heads * blocks_of(n_heads / n_kv_heads), max_len);
  const double own_bytes = (double)B * max_len * n_kv_heads * head_dim * (kv_type == kKvBf16 ? 4 : 2);
  if (n_groups > 0) {
    p.prefix = prefix_splits(B, n_heads, n_kv_heads, n_groups, max_prefix, own_bytes);
    p.joined = joined_of(p.prefix, B, n_heads, n_kv_heads, head_dim, kv_type, max_len, max_prefix, own_bytes);
  }
  return p;
}
int tile_most_states(int B, int n_heads, int n_kv_heads, int max_len, int max_prefix) {
  return tile_splits((long)B * n_kv_heads * blocks_of(n_heads / n_kv_heads), max_len) +
         (max_prefix > 0 ? prefix_splits(B, n_heads, n_kv_heads, 1, max_prefix, 0.0) : 0);
}
size_t tile_states_bytes(int B, int n_heads, int head_dim, int states) {
  return states <= 1 ? 0 : (size_t)B * n_heads * states * (head_dim + kStatePad) * sizeof(float);
}

template <int HD, int T>
static hipError_t launch_tiles(const TileAttention& t, hipStream_t stream) {
  const int G = t.n_heads / t.n_kv_heads;
  TileArgs a{};
  a.q = (const uint16_t*)t.q; a.q_stride = t.q_stride;
  a.k = t.cache.k; a.v = t.cache.v;
  a.k_scale = (const uint16_t*)t.cache.k_scale; a.v_scale = (const uint16_t*)t.cache.v_scale;
  a.n_heads = t.n_heads; a.n_kv_heads = t.n_kv_heads;
  a.scale_log2e = 1.4426950408889634f / sqrtf((float)HD);
  a.n_states = t.plan.joined ? 1 : t.plan.prefix + t.plan.own;
  a.o = (uint16_t*)t.o; a.partial = (float*)t.states;
  long blocks = 0;
  auto part = [&](TilePart& p, const int32_t* cu, const int32_t* lens, const int32_t* tables, int len_add, int max_pages,
                  int groups, long cols, long max_len, int splits, int first_state) {
    const long pages = (max_len + kKvPage - 1) / kKvPage;
    p.cu_rows = cu; p.lens = lens; p.tables = tables;
    p.len_add = len_add; p.max_len = (int)max_len; p.max_pages = max_pages; p.groups = groups;
    p.wide = cols > kNarrowCols;
    p.solo = !p.wide && solo_of((long)groups * t.n_kv_heads, max_len);
    p.blocks_x = p.solo ? (t.n_kv_heads + kTileWaves - 1) / kTileWaves : t.n_kv_heads * blocks_of(cols);
    p.splits = splits;
    p.pages_per_split = !cu && t.plan.cut && splits > 1 ? 0 : (int)((pages + splits - 1) / splits);
    p.first_state = first_state;
    blocks += (long)p.blocks_x * groups * splits;
  };
  const bool joined = t.plan.joined;
  if (joined) {
    TilePart& p = a.part[0];
    p.cu_rows = t.cu_groups; p.lens = t.prefix_lens; p.tables = t.prefix_tables;
    p.max_len = t.max_prefix; p.max_pages = t.max_prefix_pages; p.groups = t.n_groups;
  } else if (t.plan.prefix > 0) {
    part(a.part[0], t.cu_groups, t.prefix_lens, t.prefix_tables, 0, t.max_prefix_pages, t.n_groups, (long)t.max_rows * G,
         t.max_prefix, t.plan.prefix, 0);
    a.first_blocks = (int)blocks;
  }
  part(a.part[1], nullptr, t.kv_lens, t.block_tables, t.kv_len_add, t.max_blocks, t.B, G,
       joined ? (long)t.max_kv_len + t.max_prefix : t.max_kv_len, joined ? 1 : t.plan.own, joined ? 0 : t.plan.prefix);
  a.part[1].max_len = t.max_kv_len;
  a.part[1].rank = t.B > 1;
  const bool wide = a.part[0].wide || a.part[1].wide;
  const bool once = (double)t.B * t.max_kv_len * t.n_kv_heads * HD * (T == kKvBf16 ? 4 : 2) > kOnceBytes;
  const dim3 grid((unsigned)blocks), threads(kTileThreads);
  if (joined) {
    hipLaunchKernelGGL((tile_attention_kernel<HD, T, false, false, true>), grid, threads, 0, stream, a);
  } else if (T == kKvBf16 || wide) {
    if (once) hipLaunchKernelGGL((tile_attention_kernel<HD, T, true, true, false>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((tile_attention_kernel<HD, T, true, false, false>), grid, threads, 0, stream, a);
  } else if constexpr (T != kKvBf16) {
    if (once) hipLaunchKernelGGL((tile_attention_kernel<HD, T, false, true, false>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((tile_attention_kernel<HD, T, false, false, false>), grid, threads, 0, stream, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_states == 1) return e;
  // Few states: a wave is enough for them, and a quarter of the workgroups (2560 of up to 9 states 5.6 -> 4.7 us).
  const int items = t.B * t.n_heads;
  if (a.n_states <= kTileWaves * 8)
    hipLaunchKernelGGL((tile_combine_kernel<HD, 1>), dim3((items + kTileWaves - 1) / kTileWaves), threads, 0, stream, a.partial,
                       items, a.n_states, t.plan.cut ? t.plan.prefix : -1, a.o);
  else
    hipLaunchKernelGGL((tile_combine_kernel<HD, kTileWaves>), dim3(items), threads, 0, stream, a.partial, items, a.n_states,
                       t.plan.cut ? t.plan.prefix : -1, a.o);
  return hipGetLastError();
}

bool tile_attention_fits(const TileAttention& t) {
  const int G = t.n_heads / t.n_kv_heads;
  const double own = (double)t.B * blocks_of(G) * t.plan.own;
  const double prefixes = t.plan.joined ? 0.0 : (double)t.n_groups * blocks_of((long)t.max_rows * G) * t.plan.prefix;
  return t.B <= 65535 && (own + prefixes) * t.n_kv_heads <= (double)(0x7fffffff / kTileThreads);
}

hipError_t launch_tile_attention(const TileAttention& t, hipStream_t stream) {
  if (t.n_kv_heads <= 0 || t.n_heads % t.n_kv_heads != 0 || !tile_attention_fits(t)) return hipErrorInvalidValue;
  if (t.plan.own < 1 || (t.plan.own + t.plan.prefix > 1 && !t.states)) return hipErrorInvalidValue;
  if (t.head_dim == 128) {
    if (t.cache.type == kKvBf16) return launch_tiles<128, kKvBf16>(t, stream);
    if (t.cache.type == kKvE4m3) return launch_tiles<128, kKvE4m3>(t, stream);
    if (t.cache.type == kKvInt8) return launch_tiles<128, kKvInt8>(t, stream);
  } else if (t.head_dim == 64) {
    if (t.cache.type == kKvBf16) return launch_tiles<64, kKvBf16>(t, stream);
    if (t.cache.type == kKvE4m3) return launch_tiles<64, kKvE4m3>(t, stream);
    if (t.cache.type == kKvInt8) return launch_tiles<64, kKvInt8>(t, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace ds
