// New rows of Q, K and V on their way from the QKV product: Q and K turned by their positions, K and V into the paged cache.
//
// A pair (a, b) of a head's features at position p becomes (a cos - b sin, b cos + a sin), cos and sin from row p of a table.  In
// fp32, products and sums rounded one by one (no fused multiply-add: the result is the definition's bit by bit, whichever of a
// pair a lane computes), then to bf16 once; a cache of 8 bits holds that bf16 row rounded again (kv_quant.h).
// Bytes bound it: every row is read once and written once or (K) twice, the table's rows come out of the caches.  12 prompts, 6800
// rows of 40 heads, into bf16 pages 84 to 92 us = 5.3 to 5.8 TB/s by card over three sets of tensors in turn, 80 over two; pieces of
// 20000 rows of 64 heads on 8 into int8 pages 136 to 141 us = 5.9 to 6.2 (a copy reaches 5.1).  One row of 64 sequences of 64 heads on 8: 3.8 us on the GPU, 5.2
// from call to call, which is the host.
//
// A launch has up to two parts:
//  * rows: a wave has 4 rows, 16 lanes each, and some of the heads of Q, of K and, for a bf16 cache, of V.  The rows' table entries
//    stay in registers over the heads.  The other half of a pair i, i + rot / 2 is in another lane of the 16.
//  * V of 8 bits, whose pages hold a feature's 16 tokens together: a wave has a (page, head) of all its new tokens and turns
//    them in registers, or, where every sequence has one new row, 16 lanes have a (row, head) and change a byte of each piece.
#include <type_traits>

#include "kv_quant.h"

namespace ds {

constexpr int kRotThreads = 256, kRotWaves = 4;

struct RotaryArgs {
  RotaryRows r;
  KvCache cache;
  int n_heads, n_kv_heads;
  int head_blocks;   // waves that share 4 rows
  int row_waves, v_waves;
};

// The sequence of packed row r: the last that starts there or before, -1 and B where there is none; for 4 rows at once.
__device__ __forceinline__ int seq_of(const int32_t* __restrict__ cu, int B, int r0, int r) {
  const int lane = threadIdx.x & 63;
  int upto = 0;
  for (int i0 = 0; i0 <= B; i0 += 64)
    upto += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i0 + lane <= B && cu[min(i0 + lane, B)] <= r0));
  int seq = upto - 1;
  while (seq < B && cu[seq + 1] <= r) ++seq;
  return seq;
}

template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const uint16_t* p) {
  if constexpr (N == 4) {
    const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = v[j];
  } else {
    const u32x2 v = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
    w[0] = v[0];
    w[1] = v[1];
  }
}
// Rows into the pages go past the caches (V of 8 bits apart where sequences have rows of any number: its pieces, half of what
// such a cache takes, are stored as usual), and the turned rows where there are more of them than the last-level cache keeps
// for whoever reads them next.  (us, nothing past, all past, by this rule: 20000 rows of 64 heads, 320 MB of Q, 155, 141 and 141;
// 6800 of 40, 139 MB of Q and K and as much into bf16 pages, two sets of tensors in turn 95, 87 and 78, three sets 95, 88 and 91,
// and 8000 of 40 with the attention behind them 237, 234 and 230; one row of 64 sequences of 40 and its attention 115.3, 113.5
// and 113.5.)
template <int N>
__device__ __forceinline__ void store_past(void* p, const uint32_t (&w)[N]) {
  if constexpr (N == 4) __builtin_nontemporal_store(u32x4{w[0], w[1], w[2], w[3]}, reinterpret_cast<u32x4*>(p));
  else if constexpr (N == 2) __builtin_nontemporal_store(u32x2{w[0], w[1]}, reinterpret_cast<u32x2*>(p));
  else __builtin_nontemporal_store(w[0], reinterpret_cast<uint32_t*>(p));
  asm volatile("");  // (else this store and the ordinary one of another branch become a single ordinary one)
}
template <bool PAST, int N>
__device__ __forceinline__ void store_row(void* p, const uint32_t (&w)[N]) {
  if constexpr (PAST) store_past(p, w);
  else if constexpr (N == 4) st16(p, u32x4{w[0], w[1], w[2], w[3]});
  else *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[1]};
}

// What turns the E numbers of a lane: halves, E cosines and E sines (negative in the first half); adjacent, E / 2 of each.
template <int E>
struct Turn {
  float cos[E], sin[E];
  int partner;  // lane that has the other half
  bool turned;  // the lane's numbers are among the first rot

  __device__ __forceinline__ void load(const float* __restrict__ row, int rot, bool adjacent, int lane) {
    const int c = lane & 15;
    turned = c * E < rot;
    if (adjacent) {
      const int i = turned ? c * (E / 2) : 0;
#pragma unroll
      for (int j = 0; j < E / 2; j += 2) {
        const float2 x = *reinterpret_cast<const float2*>(row + i + j), y = *reinterpret_cast<const float2*>(row + rot / 2 + i + j);
        cos[j] = x.x; cos[j + 1] = x.y;
        sin[j] = y.x; sin[j + 1] = y.y;
      }
      partner = lane;
    } else {
      const int half = rot / 2 / E;  // lanes
      const bool second = c >= half;
      const int i = turned ? (second ? c - half : c) * E : 0;
      partner = turned ? (second ? lane - half : lane + half) : lane;
#pragma unroll
      for (int j = 0; j < E; j += 4) {
        const floatx4 x = *reinterpret_cast<const floatx4*>(row + i + j), y = *reinterpret_cast<const floatx4*>(row + rot / 2 + i + j);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          cos[j + k] = x[k];
          sin[j + k] = second ? y[k] : -y[k];
        }
      }
    }
  }

  __device__ __forceinline__ void apply(uint32_t (&w)[E / 2], bool adjacent) const {
#pragma clang fp contract(off)
    uint32_t r[E / 2];
    if (adjacent) {
#pragma unroll
      for (int j = 0; j < E / 2; ++j) {
        const float a = bf16_lo(w[j]), b = bf16_hi(w[j]);
        const float ac = a * cos[j], bs = b * sin[j], bc = b * cos[j], as = a * sin[j];
        r[j] = pack_bf16(ac - bs, bc + as);
      }
    } else {
#pragma unroll
      for (int j = 0; j < E / 2; ++j) {
        const uint32_t o = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * partner, (int)w[j]);
        const float x0 = bf16_lo(w[j]) * cos[2 * j], y0 = bf16_lo(o) * sin[2 * j];
        const float x1 = bf16_hi(w[j]) * cos[2 * j + 1], y1 = bf16_hi(o) * sin[2 * j + 1];
        r[j] = pack_bf16(x0 + y0, x1 + y1);
      }
    }
#pragma unroll
    for (int j = 0; j < E / 2; ++j) w[j] = turned ? r[j] : w[j];
  }
};

// 4 rows, U heads of [Q | K | V where it is bf16].  PAST: q_out and k_out past the caches.
template <int HD, int T, int U, bool PAST>
__device__ __forceinline__ void rows_part(const RotaryArgs& a, int wave) {
  constexpr int E = HD / 16;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const RotaryRows& in = a.r;
  const int r0 = wave / a.head_blocks * 4, head0 = wave % a.head_blocks * U;
  const int n = a.n_heads, n_kv = a.n_kv_heads, heads = n + (T == kKvBf16 ? 2 : 1) * n_kv;
  const int row = min(r0 + g, in.t - 1);
  bool there = r0 + g < in.t;
  uint32_t w[U][E / 2];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = min(head0 + u, heads - 1);
    const uint16_t* src = h < n ? in.q + (size_t)row * in.q_stride + (size_t)h * HD
                                : (h < n + n_kv ? in.k : in.v) + (size_t)row * in.kv_stride + (size_t)(h < n + n_kv ? h - n : h - n - n_kv) * HD;
    load_words(w[u], src + E * c);
  }
  int seq = row, at = 0;
  if (in.cu_rows) {
    seq = seq_of(in.cu_rows, in.B, min(r0, in.t - 1), row);
    there = there && seq >= 0 && seq < in.B;
    seq = min(max(seq, 0), in.B - 1);
    at = row - in.cu_rows[seq];
  }
  const int before = in.ctx_lens[seq];
  there = there && before >= 0;
  const int pos = there ? before + at : 0;
  const int turn = in.positions ? in.positions[row] : pos;
  Turn<E> t;
  t.load(in.table + (size_t)min(max(turn, 0), in.n_pos - 1) * in.rot, in.rot, in.adjacent, lane);
  size_t page = 0;
  if (there && head0 + U > n) page = (size_t)in.block_tables[(size_t)seq * in.max_blocks + pos / kKvPage] * n_kv;
  const int slot = pos % kKvPage;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = head0 + u;
    if (h >= heads) return;
    if (h < n + n_kv) t.apply(w[u], in.adjacent);
    if (h < n) {
      if (there) store_row<PAST>(in.q_out + ((size_t)row * n + h) * HD + E * c, w[u]);
      continue;
    }
    const bool is_v = h >= n + n_kv;
    const int kv = is_v ? h - n - n_kv : h - n;
    if (!is_v && in.k_out && there) store_row<PAST>(in.k_out + ((size_t)row * n_kv + kv) * HD + E * c, w[u]);
    const size_t to = (page + kv) * kKvPage + slot;
    if constexpr (T == kKvBf16) {
      if (there) store_past(static_cast<uint16_t*>(is_v ? a.cache.v : a.cache.k) + to * HD + E * c, w[u]);
    } else {
      const uint32_t sc = scale_bits<T>(row_amax(w[u]));
      const float inv = scale_inverse(sc);
      uint32_t b[E / 4];
#pragma unroll
      for (int j = 0; j < E / 4; ++j) b[j] = quantise4<T>(w[u][2 * j], w[u][2 * j + 1], sc, inv);
      if (there) {
        store_past(static_cast<uint8_t*>(a.cache.k) + to * HD + E * c, b);
        if (c == 0) static_cast<uint16_t*>(a.cache.k_scale)[to] = (uint16_t)sc;
      }
    }
  }
}

// V of 8 bits, one new row of each sequence: 16 lanes have a (row, head); a byte in each of the page's 16-byte pieces, which
// are read, changed and written whole.
template <int HD, int T>
__device__ __forceinline__ void v_bytes_part(const RotaryArgs& a, int wave, uint8_t (*rows)[HD]) {
  constexpr int E = HD / 16, W = E / 4;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, n_kv = a.n_kv_heads;
  const long item = 4l * wave + g, items = (long)a.r.t * n_kv;
  const int row = (int)(min(item, items - 1) / n_kv), kv = (int)(min(item, items - 1) % n_kv);
  const int pos = a.r.ctx_lens[row];
  const bool there = item < items && pos >= 0;
  uint32_t w[2 * W];
  load_words(w, a.r.v + (size_t)row * a.r.kv_stride + (size_t)kv * HD + E * c);
  const int slot = max(pos, 0) % kKvPage;
  size_t page = 0;
  if (there) page = (size_t)a.r.block_tables[(size_t)row * a.r.max_blocks + pos / kKvPage] * n_kv + kv;
  uint8_t* vp = static_cast<uint8_t*>(a.cache.v) + page * (HD * kKvPage) + c * kKvPage;
  u32x4 piece[E];  // of feature 16 i + c
  if (there) {
#pragma unroll
    for (int i = 0; i < E; ++i) piece[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vp + i * 16 * kKvPage));
  }
  const uint32_t sc = scale_bits<T>(row_amax(w));
  const float inv = scale_inverse(sc);
  uint8_t* mine = rows[threadIdx.x >> 4];
#pragma unroll
  for (int j = 0; j < W; ++j) *reinterpret_cast<uint32_t*>(mine + E * c + 4 * j) = quantise4<T>(w[2 * j], w[2 * j + 1], sc, inv);
  __builtin_amdgcn_wave_barrier();  // (16 lanes of one wave exchange the row)
  if (!there) return;
  if (c == 0) static_cast<uint16_t*>(a.cache.v_scale)[page * kKvPage + slot] = (uint16_t)sc;
  const uint32_t shift = 8 * (slot & 3);
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const uint32_t v = (uint32_t)mine[16 * i + c] << shift;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q == slot >> 2) piece[i][q] = (piece[i][q] & ~(0xffu << shift)) | v;
    __builtin_nontemporal_store(piece[i], reinterpret_cast<u32x4*>(vp + i * 16 * kKvPage));
  }
}

// V of 8 bits, rows of sequences: a wave has the new tokens of a (page, head).  Sequence i has the places cu[i] / 16 + 2 i and on:
// its rows lie in at most rows / 16 + 2 pages, wherever in a page they begin, and there are t / 16 + 2 B places in all.
template <int HD, int T>
__device__ __forceinline__ void v_pages_part(const RotaryArgs& a, int wave) {
  constexpr int E = HD / 16, W = E / 4;
  const RotaryRows& in = a.r;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, n_kv = a.n_kv_heads;
  const int place = wave / n_kv, kv = wave % n_kv;
  int upto = 0;  // sequences that begin here or before
  for (int i0 = 0; i0 < in.B; i0 += 64) {
    const int i = i0 + lane;
    upto += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i < in.B && in.cu_rows[min(i, in.B - 1)] / kKvPage + 2 * i <= place));
  }
  if (upto == 0) return;
  const int seq = upto - 1, start = in.cu_rows[seq], count = min(in.cu_rows[seq + 1], in.t) - start, before = in.ctx_lens[seq];
  if (before < 0 || count <= 0) return;
  const int at = before / kKvPage + place - start / kKvPage - 2 * seq, tok0 = at * kKvPage;  // the page, its first token
  const int lo = max(before - tok0, 0), hi = min(before + count - tok0, kKvPage);            // its new slots
  if (hi <= lo) return;
  PageRows<HD> rows;
  rows.load(in.v + ((ptrdiff_t)start + tok0 - before) * in.kv_stride + (size_t)kv * HD, in.kv_stride, g, c, hi - 1, lo);
  __builtin_amdgcn_sched_barrier(0);  // the page's number is not waited for before the loads are out
  const size_t page = (size_t)in.block_tables[(size_t)seq * in.max_blocks + at] * n_kv + kv;
  uint32_t sc[4], out[W][4];  // out[j][i]: values 4 j .. 4 j + 3 of the lane's E, token 4 g + i
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sc[i] = scale_bits<T>(row_amax(rows.w[i]));
    const float inv = scale_inverse(sc[i]);
#pragma unroll
    for (int j = 0; j < W; ++j) out[j][i] = quantise4<T>(rows.w[i][2 * j], rows.w[i][2 * j + 1], sc[i], inv);
  }
  const int mine = 4 * g + c;
  if (c < 4 && mine >= lo && mine < hi)
    static_cast<uint16_t*>(a.cache.v_scale)[page * kKvPage + mine] = (uint16_t)(c == 0 ? sc[0] : c == 1 ? sc[1] : c == 2 ? sc[2] : sc[3]);
  uint32_t f[E];
  turn_page<HD>(out, f);
  uint8_t* dst = static_cast<uint8_t*>(a.cache.v) + page * (kKvPage * HD) + (E * c + W * g) * kKvPage;
#pragma unroll
  for (int e = 0; e < W; ++e) {  // feature E c + W g + e
    u32x4 v{f[e], f[e + W], f[e + E / 2], f[e + E / 2 + W]};
    if (hi - lo < kKvPage) {  // slots that no new token has stay as they are
      const u32x4 old = ld16(dst + e * kKvPage);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n0 = min(max(lo - 4 * q, 0), 4), n1 = min(max(hi - 4 * q, 0), 4);
        const uint32_t keep = (uint32_t)((1ull << (8 * n1)) - 1ull) & ~(uint32_t)((1ull << (8 * n0)) - 1ull);
        v[q] = (v[q] & keep) | (old[q] & ~keep);
      }
    }
    st16(dst + e * kKvPage, v);
  }
}

template <int HD, int T, int U, bool PAST>
__global__ __launch_bounds__(kRotThreads) void kv_append_rotary_kernel(const RotaryArgs a) {
  const int wave = (int)blockIdx.x * kRotWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (wave < a.row_waves) return rows_part<HD, T, U, PAST>(a, wave);
  if constexpr (T != kKvBf16) {
    __shared__ __attribute__((aligned(16))) uint8_t rows[kRotThreads / 16][HD];
    if (wave >= a.row_waves + a.v_waves) return;
    if (a.r.cu_rows) v_pages_part<HD, T>(a, wave - a.row_waves);
    else v_bytes_part<HD, T>(a, wave - a.row_waves, rows);
  }
}

constexpr double kKeptBytes = 200e6;  // what is left of the last-level cache beside what is read

// Heads of a wave, where that leaves two waves a SIMD or more; else 1.  (8: the 6800 rows above, three sets of tensors in turn, 94.3
// instead of 91.9 us, the 20000 144.4 instead of 141.2.)
constexpr int kHeads = 4;

struct RotaryPlan {
  int heads;
  long head_blocks, row_waves, v_waves;
};
static RotaryPlan rotary_plan(const RotaryRows& r, int kv_type, int n_heads, int n_kv_heads) {
  RotaryPlan p;
  const long heads = n_heads + (kv_type == kKvBf16 ? 2l : 1l) * n_kv_heads, groups = ((long)r.t + 3) / 4;
  p.heads = groups * ((heads + kHeads - 1) / kHeads) < 2048 ? 1 : kHeads;
  p.head_blocks = (heads + p.heads - 1) / p.heads;
  p.row_waves = groups * p.head_blocks;
  p.v_waves = kv_type == kKvBf16 ? 0
              : r.cu_rows        ? ((long)r.t / kKvPage + 2l * r.B) * n_kv_heads
                                 : ((long)r.t * n_kv_heads + 3) / 4;
  return p;
}
static long rotary_blocks(const RotaryPlan& p) { return (p.row_waves + p.v_waves + kRotWaves - 1) / kRotWaves; }

bool rotary_fits(const RotaryRows& r, int kv_type, int n_heads, int n_kv_heads) {
  return rotary_blocks(rotary_plan(r, kv_type, n_heads, n_kv_heads)) <= 0x7fffffffL / kRotThreads;
}

hipError_t launch_kv_append_rotary(const RotaryRows& r, const KvCache& cache, int n_heads, int n_kv_heads, int head_dim,
                                   hipStream_t stream) {
  if (!rotary_fits(r, cache.type, n_heads, n_kv_heads)) return hipErrorInvalidValue;
  const RotaryPlan p = rotary_plan(r, cache.type, n_heads, n_kv_heads);
  const RotaryArgs a{r, cache, n_heads, n_kv_heads, (int)p.head_blocks, (int)p.row_waves, (int)p.v_waves};
  const bool past = 2.0 * r.t * head_dim * (n_heads + (r.k_out ? n_kv_heads : 0)) > kKeptBytes;
  const dim3 grid((unsigned)rotary_blocks(p)), threads(kRotThreads);
  using std::integral_constant;
  auto sized = [&](auto hd, auto type) {
    if (p.heads == 1) hipLaunchKernelGGL((kv_append_rotary_kernel<hd(), type(), 1, false>), grid, threads, 0, stream, a);
    else if (past) hipLaunchKernelGGL((kv_append_rotary_kernel<hd(), type(), kHeads, true>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((kv_append_rotary_kernel<hd(), type(), kHeads, false>), grid, threads, 0, stream, a);
    return hipGetLastError();
  };
  auto typed = [&](auto hd) {
    if (cache.type == kKvBf16) return sized(hd, integral_constant<int, kKvBf16>{});
    if (cache.type == kKvE4m3) return sized(hd, integral_constant<int, kKvE4m3>{});
    if (cache.type == kKvInt8) return sized(hd, integral_constant<int, kKvInt8>{});
    return hipErrorInvalidValue;
  };
  if (head_dim == 128) return typed(integral_constant<int, 128>{});
  if (head_dim == 64) return typed(integral_constant<int, 64>{});
  return hipErrorInvalidValue;
}

}  // namespace ds
