// Attention of single queries over pages in tiles of the matrix cores: over the paged cache of 8 bits, and over a prefix
// whose pages several sequences share (in any of the three forms of the cache).
//
// The 16 columns of a tile are queries of one key/value head: the query heads that share it, of one sequence or, for a
// prefix, of all rows of the group that shares the pages.  Per 16 x 16 x 32 instruction
//   scores  S[key, column]  = K[key, :] . Q[column, :]        operand A = 16 keys, operand B = 16 columns
//   output  O^T[d, column] += V^T[d, key] . P[key, column]    operand A = 16 features, operand B = P
// In the result of the first a lane has one column (lane % 16) and 4 keys, so the softmax's running maximum and sum are
// scalars of a lane; with the keys dealt out as below the probabilities are already the second product's operand B.
//
// A workgroup of 4 waves takes one (group, key/value head, NC tiles of columns, split of the pages); its waves take turns
// by chunks of 64 (8 bits) or 32 keys (bf16), and their states (maximum, sum, output) are merged through LDS.
//   8 bits: a chunk is 4 pages, g = lane / 16 is the lane's page.  Row i of score tile t is key 4 t + i % 4 of page i / 4, so
// the lane's results are all 16 keys of page g.  V is kept with a feature's 16 tokens together: 16 bytes are the lane's
// operand for 16 keys of page g.  Values go to bf16 exactly; the scales of K multiply the scores, those of V the
// probabilities (in fp32, by a DPP operand: lane 16 g + j has the scale of key j).
//   bf16: a chunk is 2 pages, row i of score tile t is key i of page t; V goes through LDS, where the transposing read
// makes the operand.
// Probabilities are rounded to bf16 for the second product (at most 2^-9 of each, in no one direction); the sum is that of
// the unrounded ones.
#include <algorithm>
#include <type_traits>

#include "kv_quant.h"

namespace ds {

constexpr int kTileThreads = 256, kTileWaves = 4;

struct TileArgs {
  const uint16_t* q;
  int q_stride;
  const int32_t* cu_rows;  // group i has the rows [cu_rows[i], cu_rows[i + 1]); null: row i
  const int32_t* lens;
  int len_add;
  const int32_t* tables;
  int max_pages;
  const void *k, *v;
  const uint16_t *k_scale, *v_scale;
  int n_heads, n_kv_heads, pages_per_split;
  int first_state, n_states;  // a (row, head) has n_states states, this launch's from first_state on; 1: o is written
  float scale_log2e;
  uint16_t* o;
  float* partial;  // [row][head][state][max, sum, output[HD]]
};

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

template <int HD, int T>
struct Tiles {
  static constexpr bool kQuant = T != kKvBf16;
  static constexpr int kPages = kQuant ? 4 : 2;       // of a chunk
  static constexpr int kTilesS = kPages;              // score tiles of 16 keys
  static constexpr int kSteps = HD / 32;              // instructions per score tile
  static constexpr int kVRow = HD + 16;               // LDS row of a staged V page (bf16): 8 banks further than the last
  static constexpr int kStage = kQuant ? 0 : 2 * kKvPage * kVRow * 2;  // bytes of a wave
  static constexpr int kMerge = kTileWaves * 16 * (HD + 2) * 4;
  static constexpr int kLds = kTileWaves * kStage > kMerge ? kTileWaves * kStage : kMerge;
};

template <int HD, int T, int NC>
__global__ __launch_bounds__(kTileThreads) __attribute__((amdgpu_waves_per_eu(2))) void tile_attention_kernel(
    const TileArgs a) {
  using C = Tiles<HD, T>;
  constexpr int DB = HD / 16;
  __shared__ __attribute__((aligned(16))) unsigned char smem[C::kLds];
  const int G = a.n_heads / a.n_kv_heads;
  const int kv = blockIdx.x % a.n_kv_heads, c0 = blockIdx.x / a.n_kv_heads * (16 * NC);
  const int group = blockIdx.y, split = blockIdx.z;
  const int row0 = a.cu_rows ? a.cu_rows[group] : group;
  const int cols = (a.cu_rows ? a.cu_rows[group + 1] - row0 : 1) * G;
  if (c0 >= cols) return;
  const int tid = threadIdx.x, lane = tid & 63, hl = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = a.lens[group] + a.len_add;
  const int n_pages = (len + kKvPage - 1) / kKvPage;
  const int page_lo = split * a.pages_per_split, page_hi = min(n_pages, page_lo + a.pages_per_split);
  const int32_t* bt = a.tables + (size_t)group * a.max_pages;

  // operand B of the scores.  8 bits: instruction 2 c + h takes features 64 c + 16 g + 8 h .. + 8 of lane group g (16 bytes of
  // K are two operands); bf16: instruction s features 32 s + 8 g .. + 8.
  u32x4 qf[NC][C::kSteps];
#pragma unroll
  for (int t = 0; t < NC; ++t) {
    const int col = c0 + 16 * t + hl;
    const uint16_t* qp = a.q + (size_t)(row0 + col / G) * a.q_stride + (size_t)(kv * G + col % G) * HD;
#pragma unroll
    for (int s = 0; s < C::kSteps; ++s) {
      qf[t][s] = u32x4{0, 0, 0, 0};
      const int at = C::kQuant ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
      if (col < cols) qf[t][s] = ld16(qp + at);
    }
  }
  floatx4 acc[NC][DB];
  float m_run[NC], l_run[NC];  // l_run: this lane's share of the sum
#pragma unroll
  for (int t = 0; t < NC; ++t) {
    m_run[t] = -INFINITY;
    l_run[t] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[t][db] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  // Softmax over a chunk's scores (scaled, -inf where there is no key): new maximum, old results rescaled, p in place of s.
  auto softmax = [&](int t, auto& s) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < C::kTilesS; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) top = fmaxf(top, s[i][r]);
    top = across_groups<16>(top, MaxOp());
    const float m_new = fmaxf(m_run[t], top);
    const float alpha = __builtin_amdgcn_exp2f(m_run[t] - m_new);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < C::kTilesS; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[i][r] = __builtin_amdgcn_exp2f(s[i][r] - m_new);
        sum += s[i][r];
      }
    l_run[t] = l_run[t] * alpha + sum;
    m_run[t] = m_new;
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[t][db] *= alpha;
  };

  if constexpr (C::kQuant) {
    const uint8_t* kc = static_cast<const uint8_t*>(a.k);
    const uint8_t* vc = static_cast<const uint8_t*>(a.v);
    constexpr int KL = HD / 64;  // 16-byte loads of a key per lane
    for (int pg = page_lo + 4 * wave; pg < page_hi; pg += 4 * kTileWaves) {
      // pages of the lane: hl / 4 as a row of K, g as a column of V (behind the last: the last again, without keys)
      const size_t kp = (size_t)bt[min(pg + (hl >> 2), page_hi - 1)] * a.n_kv_heads + kv;
      const size_t vp = (size_t)bt[min(pg + g, page_hi - 1)] * a.n_kv_heads + kv;
      const int there = pg + g < page_hi ? min(len - (pg + g) * kKvPage, kKvPage) : 0;  // keys of the lane's page
      u32x4 kr[4][KL], vr[DB];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int c = 0; c < KL; ++c) kr[t][c] = ld16(kc + (kp * kKvPage + 4 * t + (hl & 3)) * HD + 64 * c + 16 * g);
#pragma unroll
      for (int db = 0; db < DB; ++db) vr[db] = ld16(vc + (vp * HD + 16 * db + hl) * kKvPage);
      const float ks = bf16_lo(a.k_scale[vp * kKvPage + hl]) * a.scale_log2e;
      const float vs = hl < there ? bf16_lo(a.v_scale[vp * kKvPage + hl]) : 0.f;

      floatx4 s[NC][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int n = 0; n < NC; ++n) s[n][t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KL; ++c)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const u32x2 lo = values4<T>(kr[t][c][2 * h]), hi = values4<T>(kr[t][c][2 * h + 1]);
            const u32x4 kf = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
            for (int n = 0; n < NC; ++n) s[n][t] = mfma(kf, qf[n][2 * c + h], s[n][t]);
          }
      }
      u32x4 pf[NC][2];
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        each(std::make_integer_sequence<int, 16>{}, [&](auto j) {
          const float x = s[n][j() / 4][j() % 4] * row_lane<j()>(ks);
          s[n][j() / 4][j() % 4] = j() < there ? x : -INFINITY;  // (whatever the slot holds)
        });
        softmax(n, s[n]);
        each(std::make_integer_sequence<int, 16>{}, [&](auto j) { s[n][j() / 4][j() % 4] *= row_lane<j()>(vs); });
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int w = 0; w < 4; ++w)
            pf[n][h][w] = pack_bf16(s[n][2 * h + w / 2][2 * (w % 2)], s[n][2 * h + w / 2][2 * (w % 2) + 1]);
      }
      // slots behind the end may hold NaN, and 0 * NaN is NaN
      u32x4 keep;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int n = min(max(there - 4 * w, 0), 4);
        keep[w] = n == 4 ? 0xffffffffu : (1u << (8 * n)) - 1u;
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const u32x4 v = vr[db] & keep;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const u32x2 lo = values4<T>(v[2 * h]), hi = values4<T>(v[2 * h + 1]);
          const u32x4 vf = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
          for (int n = 0; n < NC; ++n) acc[n][db] = mfma(vf, pf[n][h], acc[n][db]);
        }
      }
    }
  } else {
    const uint16_t* kc = static_cast<const uint16_t*>(a.k);
    const uint16_t* vc = static_cast<const uint16_t*>(a.v);
    uint16_t* vst = reinterpret_cast<uint16_t*>(smem + wave * C::kStage);
    constexpr int CPR = HD / 8, RPL = 64 / CPR;  // 16-byte pieces of a row, rows of a load
    constexpr int NL = kKvPage / RPL;            // loads of a page
    const int vrow = lane / CPR, vcol = lane % CPR * 8;
    for (int pg = page_lo + 2 * wave; pg < page_hi; pg += 2 * kTileWaves) {
      u32x4 kr[2][C::kSteps], vr[2][NL];
      int there[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const size_t p = ((size_t)bt[min(pg + u, page_hi - 1)] * a.n_kv_heads + kv) * (kKvPage * HD);
        there[u] = pg + u < page_hi ? min(len - (pg + u) * kKvPage, kKvPage) : 0;
#pragma unroll
        for (int s = 0; s < C::kSteps; ++s) kr[u][s] = ld16(kc + p + hl * HD + 32 * s + 8 * g);
#pragma unroll
        for (int i = 0; i < NL; ++i) vr[u][i] = ld16(vc + p + (size_t)(RPL * i + vrow) * HD + vcol);
      }
      floatx4 s[NC][2];
#pragma unroll
      for (int n = 0; n < NC; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          s[n][u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int st = 0; st < C::kSteps; ++st) s[n][u] = mfma(kr[u][st], qf[n][st], s[n][u]);
        }
      // (rows behind the end as zeros: what is there may be NaN, and 0 * NaN is NaN)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const int row = RPL * i + vrow;
          *reinterpret_cast<u32x4*>(vst + (u * kKvPage + row) * C::kVRow + vcol) = row < there[u] ? vr[u][i] : u32x4{0, 0, 0, 0};
        }
      u32x4 pf[NC];
#pragma unroll
      for (int n = 0; n < NC; ++n) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[n][u][r] = 4 * g + r < there[u] ? s[n][u][r] * a.scale_log2e : -INFINITY;
        softmax(n, s[n]);
#pragma unroll
        for (int w = 0; w < 4; ++w) pf[n][w] = pack_bf16(s[n][w / 2][2 * (w % 2)], s[n][w / 2][2 * (w % 2) + 1]);
      }
      __builtin_amdgcn_wave_barrier();  // (a wave's LDS accesses keep their order; the compiler has to keep it too)
      // lane i of a group of 16 hands in 4 features of key 4 g + i / 4 and is handed 4 keys of feature i
      typedef short short4v __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) short4v* lds_short4_ptr;
      const uint16_t* vfrag = vst + (4 * g + (hl >> 2)) * C::kVRow + (hl & 3) * 4;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const u32x2 p0 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_ptr)(vfrag + 16 * db)));
        const u32x2 p1 = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_ptr)(vfrag + kKvPage * C::kVRow + 16 * db)));
        const u32x4 vf = {p0[0], p0[1], p1[0], p1[1]};
#pragma unroll
        for (int n = 0; n < NC; ++n) acc[n][db] = mfma(vf, pf[n], acc[n][db]);
      }
      __builtin_amdgcn_wave_barrier();
    }
  }

  // Merge the waves, a tile of columns at a time.  A wave without keys has maximum -inf and weight 0.
  float* mg = reinterpret_cast<float*>(smem);  // [wave][column][max, sum, output[HD]]
#pragma unroll
  for (int t = 0; t < NC; ++t) {
    const float l = across_groups<16>(l_run[t], AddOp());
    __syncthreads();  // the staging areas, or the tile before, are done with
    float* dst = mg + (size_t)(wave * 16 + hl) * (HD + 2);
    if (g == 0) {
      dst[0] = m_run[t];
      dst[1] = l;
    }
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 4; ++r) dst[2 + 16 * db + 4 * g + r] = acc[t][db][r];
    __syncthreads();
    constexpr int ND = HD / 16;
    const int col = c0 + 16 * t + (tid >> 4), d0 = (tid & 15) * ND;
    if (col < cols) {
      float m = -INFINITY, sum = 0.f, out[ND];
#pragma unroll
      for (int w = 0; w < kTileWaves; ++w) m = fmaxf(m, mg[(size_t)(w * 16 + (tid >> 4)) * (HD + 2)]);
#pragma unroll
      for (int j = 0; j < ND; ++j) out[j] = 0.f;
#pragma unroll
      for (int w = 0; w < kTileWaves; ++w) {
        const float* src = mg + (size_t)(w * 16 + (tid >> 4)) * (HD + 2);
        const float f = src[0] > -INFINITY ? __builtin_amdgcn_exp2f(src[0] - m) : 0.f;  // (NaN: its sum and output are NaN, times anything)
        sum += src[1] * f;
#pragma unroll
        for (int j = 0; j < ND; ++j) out[j] += src[2 + d0 + j] * f;
      }
      const size_t item = (size_t)(row0 + col / G) * a.n_heads + kv * G + col % G;
      if (a.n_states == 1) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;  // no key at all: 0
        uint32_t w[ND / 2];
#pragma unroll
        for (int j = 0; j < ND / 2; ++j) w[j] = pack_bf16(out[2 * j] * inv, out[2 * j + 1] * inv);
        uint16_t* op = a.o + item * HD + d0;
        if constexpr (ND == 8) st16(op, u32x4{w[0], w[1], w[2], w[3]});
        else *reinterpret_cast<u32x2*>(op) = u32x2{w[0], w[1]};
      } else {
        float* st = a.partial + (item * a.n_states + a.first_state + split) * (HD + 2);
        if ((tid & 15) == 0) {
          st[0] = m;
          st[1] = sum;
        }
#pragma unroll
        for (int j = 0; j < ND; ++j) st[2 + d0 + j] = out[j];
      }
    }
  }
}

// The states of a (row, head) as one, in their order: the same bits whenever.
template <int HD>
__global__ __launch_bounds__(HD) void tile_combine_kernel(const float* __restrict__ partial, int n_states,
                                                          uint16_t* __restrict__ o) {
  const size_t item = blockIdx.x;
  const float* src = partial + item * n_states * (HD + 2);
  float m = -INFINITY, sum = 0.f, out = 0.f;
  for (int s = 0; s < n_states; ++s) m = fmaxf(m, src[(size_t)s * (HD + 2)]);
  for (int s = 0; s < n_states; ++s) {
    const float* st = src + (size_t)s * (HD + 2);
    const float f = st[0] > -INFINITY ? __builtin_amdgcn_exp2f(st[0] - m) : 0.f;
    sum += st[1] * f;
    out += st[2 + threadIdx.x] * f;
  }
  reinterpret_cast<__bf16*>(o)[item * HD + threadIdx.x] = (__bf16)(sum == 0.f ? 0.f : out / sum);
}

// ---- plans ----
// Column tiles of a workgroup.
static int column_tiles(long cols) { return cols <= 16 ? 1 : 2; }

// Splits of up to max_len tokens for `columns` queries of each key/value head in all: enough for two workgroups per compute
// unit, of 16 pages or more.  (Of a prefix: as though one group had all rows.)
static int tile_splits(long columns, int n_kv_heads, int max_len) {
  const int nc = column_tiles(columns);
  const long items = n_kv_heads * ((columns + 16 * nc - 1) / (16 * nc));
  const int pages = (max_len + kKvPage - 1) / kKvPage;
  const long wanted = (512 + items - 1) / items;
  return (int)std::max(1l, std::min(wanted, (long)pages / 16));
}

TilePlan tile_plan(int B, int n_heads, int n_kv_heads, int max_len, int max_prefix) {
  const int G = n_heads / n_kv_heads;
  TilePlan p;
  p.own = tile_splits(16l * B * ((G + 15) / 16), n_kv_heads, max_len);
  p.prefix = max_prefix > 0 ? tile_splits((long)B * G, n_kv_heads, max_prefix) : 0;
  return p;
}
size_t tile_states_bytes(int B, int n_heads, int head_dim, int states) {
  return states <= 1 ? 0 : (size_t)B * n_heads * states * (head_dim + 2) * sizeof(float);
}

template <int HD, int T>
static hipError_t launch_tiles(TileArgs a, int groups, long cols, int max_len, int splits, hipStream_t stream) {
  const int nc = column_tiles(cols);
  const long blocks = (cols + 16 * nc - 1) / (16 * nc) * a.n_kv_heads;
  const int pages = (max_len + kKvPage - 1) / kKvPage;
  a.pages_per_split = (pages + splits - 1) / splits;
  if (blocks > 0x7fffffffL / kTileThreads || groups > 65535 || splits > 65535) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks, groups, splits), threads(kTileThreads);
  if (nc == 1) hipLaunchKernelGGL((tile_attention_kernel<HD, T, 1>), grid, threads, 0, stream, a);
  else hipLaunchKernelGGL((tile_attention_kernel<HD, T, 2>), grid, threads, 0, stream, a);
  return hipGetLastError();
}

template <int HD, int T>
static hipError_t launch_all(const TileAttention& t, hipStream_t stream) {
  TileArgs a{};
  a.q = (const uint16_t*)t.q; a.q_stride = t.q_stride;
  a.k = t.cache.k; a.v = t.cache.v;
  a.k_scale = (const uint16_t*)t.cache.k_scale; a.v_scale = (const uint16_t*)t.cache.v_scale;
  a.n_heads = t.n_heads; a.n_kv_heads = t.n_kv_heads;
  a.scale_log2e = 1.4426950408889634f / sqrtf((float)HD);
  a.n_states = t.plan.prefix + t.plan.own;
  a.o = (uint16_t*)t.o; a.partial = (float*)t.states;
  const int G = t.n_heads / t.n_kv_heads;
  if (t.plan.prefix > 0) {
    a.cu_rows = t.cu_groups; a.lens = t.prefix_lens; a.tables = t.prefix_tables; a.max_pages = t.max_prefix_pages;
    a.first_state = 0;
    const hipError_t e = launch_tiles<HD, T>(a, t.n_groups, (long)t.max_rows * G, t.max_prefix, t.plan.prefix, stream);
    if (e != hipSuccess) return e;
  }
  a.cu_rows = nullptr; a.lens = t.kv_lens; a.len_add = t.kv_len_add; a.tables = t.block_tables; a.max_pages = t.max_blocks;
  a.first_state = t.plan.prefix;
  hipError_t e = launch_tiles<HD, T>(a, t.B, G, t.max_kv_len, t.plan.own, stream);
  if (e != hipSuccess || a.n_states == 1) return e;
  hipLaunchKernelGGL(tile_combine_kernel<HD>, dim3(t.B * t.n_heads), dim3(HD), 0, stream, a.partial, a.n_states, a.o);
  return hipGetLastError();
}

hipError_t launch_tile_attention(const TileAttention& t, hipStream_t stream) {
  if (t.n_kv_heads <= 0 || t.n_heads % t.n_kv_heads != 0 || t.B > 65535) return hipErrorInvalidValue;
  if (t.plan.own < 1 || (t.plan.own + t.plan.prefix > 1 && !t.states)) return hipErrorInvalidValue;
  if (t.head_dim == 128) {
    if (t.cache.type == kKvBf16) return launch_all<128, kKvBf16>(t, stream);
    if (t.cache.type == kKvE4m3) return launch_all<128, kKvE4m3>(t, stream);
    if (t.cache.type == kKvInt8) return launch_all<128, kKvInt8>(t, stream);
  } else if (t.head_dim == 64) {
    if (t.cache.type == kKvBf16) return launch_all<64, kKvBf16>(t, stream);
    if (t.cache.type == kKvE4m3) return launch_all<64, kKvE4m3>(t, stream);
    if (t.cache.type == kKvInt8) return launch_all<64, kKvInt8>(t, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace ds
