// The paged cache of 8 bits as it is written (hand-off, append) and read back.  Formats and layout: kv_quant.h.
// All three move bytes: what has to be read and written bounds them.  12 ragged prompts of 40 heads, 5197 tokens, int8: 160 MB
// written off in 30 us (5.4 TB/s) and read back in 26 (6.3: that much stays in the last-level cache); 8 of 2048, 96 heads, e4m3,
// one behind the other: 1.2 GB in 195 and back in 252 us (6.2 and 4.8, together 5.4 TB/s; a large copy reaches 5.15 here).
#include <type_traits>

#include "kv_quant.h"

namespace ds {

constexpr int kQuantThreads = 256, kQuantWaves = 4;

// A wave takes one page of one head of K or of V; a workgroup 4 heads, and those of a page follow each other.
//   Sequence i has the places cu[i] / 16 + i and on, as many as it has pages or more, and there are t / 16 + B of them in all:
// next to none is for nothing, however unlike the lengths are.  (A grid of the longest sequence's pages times sequences took 8 us
// more either way for the 12 prompts.)
struct PagePlace {
  int seq, page, head, ntok;
  size_t row0;  // of the page's first token
  bool v, none;
};
__device__ __forceinline__ PagePlace page_place(const int32_t* __restrict__ cu_seqlens, int B, int max_seqlen, int n_heads) {
  PagePlace p;
  const int groups = (n_heads + kQuantWaves - 1) / kQuantWaves;
  const int place = blockIdx.x / (2 * groups), part = blockIdx.x % (2 * groups);
  p.v = part >= groups;
  p.head = (p.v ? part - groups : part) * kQuantWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int before = 0;  // sequences that start here or before
  const int lane = threadIdx.x & 63;
  for (int i0 = 0; i0 < B; i0 += 64) {
    const int i = i0 + lane;
    before += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i < B && cu_seqlens[min(i, B - 1)] / kKvPage + i <= place));
  }
  p.seq = max(before - 1, 0);
  const int start = cu_seqlens[p.seq], len = min(cu_seqlens[p.seq + 1] - start, max_seqlen);
  p.page = place - start / kKvPage - p.seq;
  const int tok0 = p.page * kKvPage;
  p.row0 = (size_t)start + tok0;
  p.ntok = min(kKvPage, len - tok0);
  p.none = before == 0 || p.page < 0 || p.ntok <= 0 || p.head >= n_heads;
  return p;
}

template <int HD, int T>
__global__ __launch_bounds__(kQuantThreads) void kv_migrate_quant_kernel(
    const uint16_t* __restrict__ k_src, const uint16_t* __restrict__ v_src, const int32_t* __restrict__ cu_seqlens, int B,
    int max_seqlen, const int32_t* __restrict__ block_tables, int max_blocks, uint8_t* __restrict__ k_cache,
    uint8_t* __restrict__ v_cache, uint16_t* __restrict__ k_scale, uint16_t* __restrict__ v_scale, int n_heads) {
  constexpr int E = HD / 16, W = E / 4;
  const PagePlace p = page_place(cu_seqlens, B, max_seqlen, n_heads);
  if (p.none) return;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const size_t h = (size_t)n_heads * HD;
  PageRows<HD> rows;
  rows.load((p.v ? v_src : k_src) + p.row0 * h + (size_t)p.head * HD, h, g, c, p.ntok - 1);
  __builtin_amdgcn_sched_barrier(0);  // the page's number is not waited for before the loads are out
  const size_t page = (size_t)block_tables[(size_t)p.seq * max_blocks + p.page] * n_heads + p.head;
  uint32_t sc[4], out[W][4];  // out[j][i]: values 4 j .. 4 j + 3 of the lane's E, token i
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sc[i] = scale_bits<T>(row_amax(rows.w[i]));
    const float inv = scale_inverse(sc[i]);
#pragma unroll
    for (int j = 0; j < W; ++j) out[j][i] = quantise4<T>(rows.w[i][2 * j], rows.w[i][2 * j + 1], sc[i], inv);
  }
  uint16_t* scales = (p.v ? v_scale : k_scale) + page * kKvPage;
  if (c < 4 && 4 * g + c < p.ntok)
    scales[4 * g + c] = (uint16_t)(c == 0 ? sc[0] : c == 1 ? sc[1] : c == 2 ? sc[2] : sc[3]);
  if (!p.v) {
    uint8_t* dst = k_cache + page * (kKvPage * HD) + E * c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (4 * g + i < p.ntok) {
        if constexpr (W == 2) *reinterpret_cast<u32x2*>(dst + (4 * g + i) * HD) = u32x2{out[0][i], out[1][i]};
        else *reinterpret_cast<uint32_t*>(dst + (4 * g + i) * HD) = out[0][i];
      }
    }
    return;
  }
  uint32_t f[E];
  turn_page<HD>(out, f);
  // tokens 0..3, 4..7, 8..11, 12..15 of feature E c + W g + e
  uint8_t* dst = v_cache + page * (kKvPage * HD) + (E * c + W * g) * kKvPage;
#pragma unroll
  for (int e = 0; e < W; ++e) {
    const uint32_t v[4] = {f[e], f[e + W], f[e + E / 2], f[e + E / 2 + W]};
    if (p.ntok == kKvPage) {
      st16(dst + e * kKvPage, u32x4{v[0], v[1], v[2], v[3]});
    } else {  // slots that no token maps to stay as they are
#pragma unroll
      for (int t = 0; t < kKvPage; ++t)
        if (t < p.ntok) dst[e * kKvPage + t] = (uint8_t)(v[t / 4] >> (8 * (t % 4)));
    }
  }
}

// The reverse: pages -> rows, each value times its scale, rounded to bf16.  The rows are stored past the caches: a head's piece of
// a row is 128 or 256 bytes and its neighbours come from other waves (the 12 prompts 37.5 -> 26.0 us).  Pages loaded or
// written (above) that way are not faster: 34.2 with the loads alone, the hand-off 29.8 -> 32.9.
template <int HD, int T>
__global__ __launch_bounds__(kQuantThreads) void kv_read_quant_kernel(
    const int32_t* __restrict__ cu_seqlens, int B, int max_seqlen, const int32_t* __restrict__ block_tables, int max_blocks,
    const uint8_t* __restrict__ k_cache, const uint8_t* __restrict__ v_cache, const uint16_t* __restrict__ k_scale,
    const uint16_t* __restrict__ v_scale, uint16_t* __restrict__ k_dst, uint16_t* __restrict__ v_dst, int n_heads) {
  constexpr int E = HD / 16, W = E / 4;
  const PagePlace p = page_place(cu_seqlens, B, max_seqlen, n_heads);
  if (p.none) return;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const size_t page = (size_t)block_tables[(size_t)p.seq * max_blocks + p.page] * n_heads + p.head;
  const u32x2 sc = *reinterpret_cast<const u32x2*>((p.v ? v_scale : k_scale) + page * kKvPage + 4 * g);
  uint32_t out[W][4];
  if (!p.v) {
    const uint8_t* src = k_cache + page * (kKvPage * HD) + E * c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (W == 2) {
        const u32x2 v = *reinterpret_cast<const u32x2*>(src + (4 * g + i) * HD);
        out[0][i] = v[0];
        out[1][i] = v[1];
      } else {
        out[0][i] = *reinterpret_cast<const uint32_t*>(src + (4 * g + i) * HD);
      }
    }
  } else {
    const uint8_t* src = v_cache + page * (kKvPage * HD) + (E * c + W * g) * kKvPage;
    uint32_t f[E];
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const u32x4 v = ld16(src + e * kKvPage);
      f[e] = v[0];
      f[e + W] = v[1];
      f[e + E / 2] = v[2];
      f[e + E / 2 + W] = v[3];
    }
#pragma unroll
    for (int e = 0; e < W; ++e) {
      swap16(f[e], f[e + W]);
      swap16(f[e + E / 2], f[e + E / 2 + W]);
    }
#pragma unroll
    for (int e = 0; e < E / 2; ++e) swap32(f[e], f[e + E / 2]);
#pragma unroll
    for (int e = 0; e < E; ++e) out[e / 4][e % 4] = f[e];
#pragma unroll
    for (int j = 0; j < W; ++j) turn_bytes(out[j]);
  }
  const size_t h = (size_t)n_heads * HD;
  uint16_t* dst = (p.v ? v_dst : k_dst) + p.row0 * h + (size_t)p.head * HD + E * c;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float cf = i & 1 ? bf16_hi(sc[i / 2]) : bf16_lo(sc[i / 2]);
    uint32_t w[2 * W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const u32x2 v = values4<T>(out[j][i]);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        // a value next to the largest bf16 may stand for more than that: not for infinity (a NaN passes)
        const float most = __uint_as_float(0x7f7f0000u);
        float lo = bf16_lo(v[k]) * cf, hi = bf16_hi(v[k]) * cf;
        lo = lo > most ? most : (lo < -most ? -most : lo);
        hi = hi > most ? most : (hi < -most ? -most : hi);
        w[2 * j + k] = pack_bf16(lo, hi);
      }
    }
    if (4 * g + i < p.ntok) {
      if constexpr (W == 2)
        __builtin_nontemporal_store(u32x4{w[0], w[1], w[2], w[3]}, reinterpret_cast<u32x4*>(dst + (size_t)(4 * g + i) * h));
      else __builtin_nontemporal_store(u32x2{w[0], w[1]}, reinterpret_cast<u32x2*>(dst + (size_t)(4 * g + i) * h));
    }
  }
}

// grid: x = sequence, y = 0: K, 1: V, z = group of 16 heads; 16 lanes take one head's row.
template <int HD, int T>
__global__ __launch_bounds__(kQuantThreads) void kv_append_quant_kernel(
    const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new, int row_stride,
    const int32_t* __restrict__ ctx_lens, const int32_t* __restrict__ block_tables, int max_blocks,
    uint8_t* __restrict__ k_cache, uint8_t* __restrict__ v_cache, uint16_t* __restrict__ k_scale,
    uint16_t* __restrict__ v_scale, int n_heads) {
  constexpr int E = HD / 16, W = E / 4;
  __shared__ __attribute__((aligned(16))) uint8_t rows[kQuantThreads / 16][HD];
  const int seq = blockIdx.x, which = blockIdx.y, c = threadIdx.x & 15;
  const int head = blockIdx.z * (kQuantThreads / 16) + (threadIdx.x >> 4);
  const int pos = ctx_lens[seq];
  if (pos < 0) return;  // a row that pads the batch
  const bool here = head < n_heads;  // (lanes of one wave exchange values: none leaves before)
  const uint16_t* src = (which ? v_new : k_new) + (size_t)seq * row_stride + (size_t)min(head, n_heads - 1) * HD + E * c;
  const int blk = block_tables[(size_t)seq * max_blocks + pos / kKvPage];
  const int slot = pos % kKvPage;
  uint32_t w[2 * W];
#pragma unroll
  for (int j = 0; j < W; ++j) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(src + 4 * j);
    w[2 * j] = v[0];
    w[2 * j + 1] = v[1];
  }
  const uint32_t sc = scale_bits<T>(row_amax(w));
  const float inv = scale_inverse(sc);
  const size_t page = (size_t)blk * n_heads + min(head, n_heads - 1);
  if (which == 0) {
    if (!here) return;
    if (c == 0) k_scale[page * kKvPage + slot] = (uint16_t)sc;
#pragma unroll
    for (int j = 0; j < W; ++j)
      *reinterpret_cast<uint32_t*>(k_cache + (page * kKvPage + slot) * HD + E * c + 4 * j) =
          quantise4<T>(w[2 * j], w[2 * j + 1], sc, inv);
    return;
  }
  // V: a byte in each of the page's 16-byte pieces.  The pieces are read, changed and written whole: written byte by byte,
  // each of the page's lines is half-masked on its way to memory (40 heads, 64 sequences 6.9 -> 5.3 us, 128 10.3 -> 7.1).  They
  // go past the caches both ways: lines left changed in an L2 are what the next launch waits for (with the attention behind
  // it, 64 sequences 75.8 -> 70.3 us, 128 117.3 -> 108.3; the stores alone past them 75.9 and 117.6, the loads alone 71.8 and
  // 116.4).
  uint8_t* vp = v_cache + page * (HD * kKvPage) + c * kKvPage;
  u32x4 piece[E];  // of feature 16 i + c
#pragma unroll
  for (int i = 0; i < E; ++i) piece[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vp + i * 16 * kKvPage));
  uint8_t* row = rows[threadIdx.x >> 4];
#pragma unroll
  for (int j = 0; j < W; ++j) *reinterpret_cast<uint32_t*>(row + E * c + 4 * j) = quantise4<T>(w[2 * j], w[2 * j + 1], sc, inv);
  __builtin_amdgcn_wave_barrier();  // (16 lanes of one wave exchange the row)
  if (!here) return;
  if (c == 0) v_scale[page * kKvPage + slot] = (uint16_t)sc;
  const uint32_t shift = 8 * (slot & 3);
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const uint32_t v = (uint32_t)row[16 * i + c] << shift;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q == slot >> 2) piece[i][q] = (piece[i][q] & ~(0xffu << shift)) | v;
    __builtin_nontemporal_store(piece[i], reinterpret_cast<u32x4*>(vp + i * 16 * kKvPage));
  }
}

// Calls f(integral constants of the head size and the type) for the instances there are.
template <class F>
static hipError_t for_instance(int head_dim, int kv_type, F&& f) {
  using std::integral_constant;
  auto typed = [&](auto hd) {
    if (kv_type == kKvE4m3) return f(hd, integral_constant<int, kKvE4m3>{});
    if (kv_type == kKvInt8) return f(hd, integral_constant<int, kKvInt8>{});
    return hipErrorInvalidValue;
  };
  if (head_dim == 128) return typed(integral_constant<int, 128>{});
  if (head_dim == 64) return typed(integral_constant<int, 64>{});
  return hipErrorInvalidValue;
}

// Workgroups for the pages of B sequences of t tokens in all; 0: more than a launch can have.
static unsigned page_blocks(int B, int t, int n_heads) {
  const long blocks = ((long)t / kKvPage + B) * 2 * ((n_heads + kQuantWaves - 1) / kQuantWaves);
  return blocks <= 0x7fffffffL / kQuantThreads ? (unsigned)blocks : 0;
}

hipError_t launch_kv_migrate_quant(const void* k_src, const void* v_src, const int32_t* cu_seqlens, int B, int t,
                                   int max_seqlen, const int32_t* block_tables, int max_blocks, const KvCache& cache,
                                   int n_heads, int head_dim, hipStream_t stream) {
  const unsigned blocks = page_blocks(B, t, n_heads);
  if (!blocks || (long)max_blocks * kKvPage < max_seqlen) return hipErrorInvalidValue;
  return for_instance(head_dim, cache.type, [&](auto hd, auto type) {
    hipLaunchKernelGGL((kv_migrate_quant_kernel<hd(), type()>), dim3(blocks), dim3(kQuantThreads), 0, stream,
                       (const uint16_t*)k_src, (const uint16_t*)v_src, cu_seqlens, B, max_seqlen, block_tables, max_blocks,
                       (uint8_t*)cache.k, (uint8_t*)cache.v, (uint16_t*)cache.k_scale, (uint16_t*)cache.v_scale, n_heads);
    return hipGetLastError();
  });
}

hipError_t launch_kv_read_quant(const int32_t* cu_seqlens, int B, int t, int max_seqlen, const int32_t* block_tables,
                                int max_blocks, const KvCache& cache, int n_heads, int head_dim, void* k_dst, void* v_dst,
                                hipStream_t stream) {
  const unsigned blocks = page_blocks(B, t, n_heads);
  if (!blocks || (long)max_blocks * kKvPage < max_seqlen) return hipErrorInvalidValue;
  return for_instance(head_dim, cache.type, [&](auto hd, auto type) {
    hipLaunchKernelGGL((kv_read_quant_kernel<hd(), type()>), dim3(blocks), dim3(kQuantThreads), 0, stream, cu_seqlens, B,
                       max_seqlen, block_tables, max_blocks, (const uint8_t*)cache.k, (const uint8_t*)cache.v,
                       (const uint16_t*)cache.k_scale, (const uint16_t*)cache.v_scale, (uint16_t*)k_dst, (uint16_t*)v_dst,
                       n_heads);
    return hipGetLastError();
  });
}

hipError_t launch_kv_append_quant(const void* k_new, const void* v_new, int row_stride, const int32_t* ctx_lens,
                                  const int32_t* block_tables, int B, int max_blocks, const KvCache& cache, int n_heads,
                                  int head_dim, hipStream_t stream) {
  const int groups = (n_heads + kQuantThreads / 16 - 1) / (kQuantThreads / 16);
  return for_instance(head_dim, cache.type, [&](auto hd, auto type) {
    hipLaunchKernelGGL((kv_append_quant_kernel<hd(), type()>), dim3(B, 2, groups), dim3(kQuantThreads), 0, stream,
                       (const uint16_t*)k_new, (const uint16_t*)v_new, row_stride, ctx_lens, block_tables, max_blocks,
                       (uint8_t*)cache.k, (uint8_t*)cache.v, (uint16_t*)cache.k_scale, (uint16_t*)cache.v_scale, n_heads);
    return hipGetLastError();
  });
}

}  // namespace ds
