// Causal attention of packed prompts through a sliding window that leaves the first tokens visible: query i sees key j <= i if
// i - j < window or j < sinks.
//
// A workgroup owns 128 rows of one key/value head, 32 a wave: a row is a (query, query head), a power of two of the heads that share
// the key/value head for each query, so that the more heads share it the fewer queries a workgroup has, and the less its windows
// reach beyond each other.  It goes over one list of keys: the first tokens before its first query's window, then from there to
// its last query.  Key number v of that list (all its rows') is seen by a row if v <= top and (v >= low or v < sinks), with
// top and low the numbers of the row's own token and of its window's first.
//
// Scores are computed transposed, S^T[key, row] = K Q^T, so that a lane holds scores of one row (lane % 32): running maximum and
// sum are scalars of a lane, and the probabilities are the column operand of O^T[d, row] = V^T P^T as they are.  K and V tiles
// of 64 keys land row-major in one of two LDS buffers by direct loads while the other is multiplied; V^T comes out through the
// transposing LDS read.
//
// 4 s operations a (query head, visible pair) bound it, and what the softmax takes beside them.  From call to call (a product of
// 8192^3 reaches 1364 TFLOP/s here, a copy 5.1 TB/s), over three sets of tensors in turn and on several cards: 64 heads on 8, one
// prompt of 16383 tokens, window 2048, 64 first ones 1.07 to 1.10 ms = 965 to 994 TFLOP/s; two of 8192, window 1024, 0.58 to 0.60 ms
// = 855 to 883; 40 heads, 12 prompts of 16 to 2048, window 256, 4 first ones, 92 to 93 us, of whose work the bytes are 54 and the
// operations 21.  Two prompts of 32 tokens of 4 heads of 64: 4.8 us, 3.8 of which any call takes.  The large ones run into the chip's power:
// with zeros for data the first takes a sixth less.  A workgroup of the third has 128 + 255 keys and a half tile of first ones: 7 tiles,
// at both ends of which there is nothing to overlap with.  A wave goes over 10 of their 13 halves, 320 keys for the 256 that each of
// its rows sees, and waits at the barriers of the others.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace ds {

constexpr int kWinWaves = 4, kWinRows = 32;  // of a workgroup, of a wave
constexpr int kWinKeys = 64;                // of a tile
constexpr float kWinSlack = 8.f;            // exponent headroom before the softmax's reference point is moved

struct WindowArgs {
  WindowRows r;
  int kv_group;      // query heads on a key/value head
  int pack_log2;     // of the heads of a row's query
  int places;        // of a head block: t / queries + B
  int blocks, per_xcd;
  float scale_log2e;
};

__device__ __forceinline__ bf16x8 as_bf16(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

template <int N>
__device__ __forceinline__ void wait_all_but() {  // vmcnt(N) alone: N in bits 3:0 and 15:14
  static_assert(N < 64);
  __builtin_amdgcn_s_waitcnt((N & 0xf) | (N >> 4) << 14 | 0x7 << 4 | 0xf << 8);
}

template <int HD>
__global__ __launch_bounds__(64 * kWinWaves) __attribute__((amdgpu_waves_per_eu(2))) void window_attention_kernel(
    const WindowArgs a) {
  constexpr int DSTEPS = HD / 16, DT = HD / 32, CPR = HD / 8;
  constexpr int TILE = kWinKeys * HD;
  constexpr int RPL = 64 / CPR;                 // tile rows of a wave-level load
  constexpr int NLD = kWinKeys / (RPL * kWinWaves);    // loads of a wave, tile and operand
  // Two buffers for K and two for V.  Each is a variable of its own, and which one an access means is known when it is compiled:
  // the compiler then sees that a load into one need not have landed before another is read.
  __shared__ __attribute__((aligned(1024))) uint16_t k_lds0[TILE], k_lds1[TILE], v_lds0[TILE], v_lds1[TILE];

  // Workgroups reach the chip's eight partitions in turn; each takes a run of the list (key/value head, place, block of its
  // heads), so that neighbours on one partition share keys.
  const int id = (blockIdx.x & 7) * a.per_xcd + (blockIdx.x >> 3);
  if (id >= a.blocks) return;
  const WindowRows& in = a.r;
  const int n_sub = a.kv_group >> a.pack_log2;
  const int sub = id % n_sub, kv = id / n_sub / a.places;
  const int place = a.places - 1 - id / n_sub % a.places;  // (late ones first: their windows are full)
  const int pack = 1 << a.pack_log2, queries = (kWinRows * kWinWaves) >> a.pack_log2;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // The sequence whose place this is: the last that begins here or before.  (Its bounds out of the lanes that looked for it: not
  // another load to wait for.)
  int seq = -1, start = 0, end = 0;
  for (int i0 = 0; i0 < in.B; i0 += 64) {
    const int i = min(i0 + lane, in.B - 1), from = in.cu_seqlens[i], upto = in.cu_seqlens[i + 1];
    const uint64_t here = __builtin_amdgcn_ballot_w64(i0 + lane < in.B && from / queries + i <= place);
    if (here == 0) break;
    const int at = 63 - __builtin_clzll(here);
    seq = i0 + at;
    start = __builtin_amdgcn_readlane(from, at);
    end = __builtin_amdgcn_readlane(upto, at);
  }
  if (seq < 0) return;
  const int len = min(end - start, in.max_seqlen);
  const int q0 = (place - start / queries - seq) * queries;
  if (q0 >= len) return;

  // the list of keys
  const int q_end = min(q0 + queries, len);
  const int band = max(q0 - in.window + 1, 0);
  // Number `first` is key `band`.  Where a wave has 32 queries and it takes no further tile, the band begins with a half tile: a
  // wave then goes over a half less (40 heads, 12 prompts, window 256, 4 first tokens, three sets of tensors in turn 95.3 -> 93.0 us,
  // one set 90.9 -> 88.6; with a tile more, one prompt of 500, window 100, one set, 13.2 -> 14.0).
  const int first_whole = min((in.sinks + 31) & ~31, band), first_least = min(in.sinks, band);
  const bool whole = a.pack_log2 == 0 && (q_end - band + first_whole + 63) / 64 == (q_end - band + first_least + 63) / 64;
  const int first = whole ? first_whole : first_least;
  const int total = q_end - band + first;
  const int n_halves = (total + 31) / 32;

  const int hl = lane >> 5, lq = lane & 31;
  const uint16_t* kbase = in.k + (size_t)start * in.k_stride + (size_t)kv * HD;
  const uint16_t* vbase = in.v + (size_t)start * in.v_stride + (size_t)kv * HD;

  // Chunk c of 16 bytes of row r of a tile lies at c ^ swizzle(r), by the source address of the load.  K (16-byte reads of 32
  // rows at one chunk number): rows of 256 bytes r & 15, of 128 bytes (r >> 1) & 7.  V (transposing 8-byte reads of 4 rows, 4
  // chunks for each half of a wave): (r & 3) << 2, ((r >> 1) & 1) << 2.
  const int ld_sub = lane / CPR, ld_c = lane % CPR;
  const int ld_row0 = wave * NLD * RPL + ld_sub;
  auto k_col = [&](int row) __attribute__((always_inline)) { return (ld_c ^ (CPR == 16 ? row & 15 : (row >> 1) & 7)) * 8; };
  const int v_col = (ld_c ^ (CPR == 16 ? ld_sub << 2 : ((ld_sub >> 1) & 1) << 2)) * 8;
  uint32_t k_off[NLD];  // bytes from the first row of a load
#pragma unroll
  for (int j = 0; j < NLD; ++j) k_off[j] = 2 * (uint32_t)(ld_sub * in.k_stride + k_col(ld_row0 + j * RPL));
  const uint32_t v_off = 2 * (uint32_t)(ld_sub * in.v_stride + v_col);
  auto to_lds = [&](const void* from, uint16_t* to) __attribute__((always_inline)) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                     (__attribute__((address_space(3))) void*)to, 16, 0, 0);
  };
  // 64 keys from number v0 on, of K or of V, into a buffer.
  auto request = [&](int v0, auto of_v, uint16_t* dst) __attribute__((always_inline)) {
    constexpr bool kV = decltype(of_v)::value;
    const uint16_t* base = kV ? vbase : kbase;
    const int stride = kV ? in.v_stride : in.k_stride;
    if (v0 >= total) return;
    dst += wave * NLD * 512;
    if ((v0 >= first || v0 + kWinKeys <= first) && v0 >= 0 && v0 + kWinKeys <= total) {  // a scalar base and 32 bits a lane
      const char* from = reinterpret_cast<const char*>(base) + 2 * (size_t)((v0 >= first ? v0 - first + band : v0) + wave * NLD * RPL) * stride;
#pragma unroll
      for (int j = 0; j < NLD; ++j) {
        uint32_t off = kV ? v_off : k_off[j];
        asm("" : "+v"(off));  // (else its sum with the base is kept for the loop, in 64 bits a lane)
        to_lds(from + 2 * (size_t)(j * RPL) * stride + off, dst + j * 512);
      }
    } else {  // (rows before the first and behind the last: those again)
#pragma unroll
      for (int j = 0; j < NLD; ++j) {
        const int row = ld_row0 + j * RPL, v = min(max(v0 + row, 0), total - 1);
        to_lds(base + (size_t)(v >= first ? v - first + band : v) * stride + (kV ? v_col : k_col(row)), dst + j * 512);
      }
    }
  };
  const std::false_type of_k;
  const std::true_type of_v;

  // the lane's rows
  const int row_q = lq >> a.pack_log2, row_head = (kv * n_sub + sub) * pack + (lq & (pack - 1));
  const int wave_q = q0 + wave * (kWinRows >> a.pack_log2);
  const bool idle = wave_q >= len;
  const int query = wave_q + row_q, top = query - band + first;
  bf16x8 qf[DSTEPS];
  {
    const uint16_t* qrow = in.q + ((size_t)start + min(query, len - 1)) * in.q_stride + (size_t)row_head * HD + hl * 8;
#pragma unroll
    for (int st = 0; st < DSTEPS; ++st) qf[st] = as_bf16(ld16(qrow + st * 16));
  }
  // Of the wave: the last number that any of its rows sees, the one up to which all do; where the first row's window begins
  // and where the last one's does.  Then the halves (of a tile: 32 keys) that any of the rows sees, [0, sink_halves) and
  // [from_half, upto_half), and those that need masks: from tail_half on, and in [sinks / 32, clear_half).
  const int wave_top = wave_q + (kWinRows >> a.pack_log2) - 1 - band + first, least_top = wave_q - band + first;
  const int wave_low = least_top - in.window + 1, most_low = wave_top - in.window + 1;
  const int sink_halves = idle ? 0 : (min(in.sinks, total) + 31) >> 5, from_half = wave_low >> 5;
  const int upto_half = idle ? 0 : min((wave_top >> 5) + 1, n_halves);
  const int tail_half = (least_top + 1) >> 5, clear_half = (most_low + 31) >> 5, seen_sinks = in.sinks >> 5;

  floatx16 oacc[DT];
  // The reference point is kept as the number that is taken off exponents, its product with the scale once rounded, and moves by
  // what these numbers differ by: scores that are equal then weigh the same before and behind a move, however far from 0 they are.
  float mb_run = kLowestScore * a.scale_log2e, l_run = 0.f;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[d][r] = 0.f;

  const int kswz = CPR == 16 ? (lq & 15) : ((lq >> 1) & 7);
  const int i16 = lane & 15;
  const int vswz = CPR == 16 ? ((i16 >> 2) << 2) : (((i16 >> 3) & 1) << 2);
  const int vchunk = 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1);
  const int k_at = lq * HD, v_at = (4 * hl + (i16 >> 2)) * HD + (i16 & 1) * 4;
  // The scores of a half tile (32 keys) are made while the half before it is brought to probabilities and multiplied with V: a
  // matrix instruction takes the matrix unit 32 cycles and its wave 4, and in the others the vector instructions go on, its own
  // wave's and those of the other wave that a SIMD has.  Each slot below is a matrix instruction, the LDS reads of one that
  // follows and a piece of the softmax, and fences keep the compiler from undoing it.
  //   A wave has 32 rows.  (64, with one wave a SIMD and half the LDS reads: their scores have to be in the accumulation registers
  // then, and are copied out of them; 64 heads on 8, 16383 tokens, window 2048 1325 us instead of 1150.  256 rows a workgroup
  // 1125 instead of 1097; three workgroups a compute unit, with 32 keys a tile in three buffers, 1131 instead of 1052, 12 prompts
  // of 40 heads 95 instead of 99.)
  float most;
  auto read_k = [&](const uint16_t* buf, int from, int st) __attribute__((always_inline)) {
    return as_bf16(ld16(buf + (k_at + ((2 * st + hl) ^ kswz) * 8 + from * HD)));
  };
  auto read_v = [&](uint16_t* buf, int from, int x, int d) __attribute__((always_inline)) {
    typedef short short4v __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) short4v* lds_short4_ptr;
    const int at = v_at + ((4 * d + vchunk) ^ vswz) * 8 + (from + x * 16) * HD;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_ptr)(buf + at)));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_ptr)(buf + (at + 8 * HD))));
    return as_bf16(u32x4{lo[0], lo[1], hi[0], hi[1]});
  };
  const floatx16 zero = {};
  bf16x2 ones;
  ones[0] = (__bf16)1.f;
  ones[1] = (__bf16)1.f;
  auto step = [&](floatx16& cur, floatx16& nxt, const uint16_t* k_buf, int k_from, uint16_t* v_buf,
                  int v_from) __attribute__((always_inline)) {
    constexpr int kOps = DSTEPS + 2 * DT;      // matrix instructions: of K, of V's first 16 keys, of its others
    constexpr int kGroup = 4;                  // operands that are read, and waited for, together
    constexpr int kFirst = 2;                  // pairs of probabilities before the first slot
    constexpr int kPairSlots = DSTEPS + DT;    // all of them are there before the slots of the last 16 keys
    bf16x8 op[kOps];
    u32x4 pw[2];  // column operands of 16 keys each
    const float mb = mb_run;
    float sum = 0.f, top_of = -INFINITY;
    auto read = [&](int f) __attribute__((always_inline)) {
      op[f] = f < DSTEPS ? read_k(k_buf, k_from, f) : read_v(v_buf, v_from, (f - DSTEPS) / DT, (f - DSTEPS) % DT);
    };
    // Probabilities 2 p and the next, rounded to bf16, 2^-8 of each at most, and a dot product of the pair with (1, 1): the sum then
    // counts the very numbers that V is multiplied by, so that a rounding which the keys have in common leaves the quotient.
    // (64 heads on 8, 16383 tokens, window 2048: 1098 us; by two additions of the unpacked halves 1132; 1108 where the compiler may
    // not put the dot products off to later slots; 1081 with the sum of the numbers before their rounding, which makes of a V that
    // is the same everywhere another.)
    auto pair = [&](int p) __attribute__((always_inline)) {
      const float p0 = __builtin_amdgcn_exp2f(cur[2 * p] * a.scale_log2e - mb);
      const float p1 = __builtin_amdgcn_exp2f(cur[2 * p + 1] * a.scale_log2e - mb);
      const uint32_t w = pack_bf16(p0, p1);
      sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), ones, sum, false);
      pw[p / 4][p % 4] = w;
    };
#pragma unroll
    for (int f = 0; f < kGroup; ++f) read(f);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int p = 0; p < kFirst; ++p) pair(p);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int slot = 0; slot < kOps; ++slot) {
      if (slot < DSTEPS) {
        nxt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[slot], qf[slot], slot == 0 ? zero : nxt, 0, 0, 0);
      } else {
        const int x = (slot - DSTEPS) / DT, d = (slot - DSTEPS) % DT;
        oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[slot], as_bf16(pw[x]), oacc[d], 0, 0, 0);
      }
      if (slot % kGroup < 2) {  // the next group's operands, half of them each time
#pragma unroll
        for (int e = 0; e < kGroup / 2; ++e) {
          const int g = (slot / kGroup + 1) * kGroup + slot % kGroup * (kGroup / 2) + e;
          if (g < kOps) read(g);
        }
      }
#pragma unroll
      for (int p = kFirst; p < 8; ++p)
        if ((p - kFirst) * kPairSlots / (8 - kFirst) == slot) pair(p);
      if (slot >= kPairSlots) {  // the maximum of the new scores in the last slots
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e * DT / 8 == slot - kPairSlots) {
            top_of = fmaxf(fmaxf(top_of, nxt[2 * e]), nxt[2 * e + 1]);
            asm volatile("" : "+v"(top_of));
          }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    l_run += sum;
    most = top_of;
  };
  // What the next half's scores still need: masks (element r is number v0 + 8 (r / 4) + 4 hl + r % 4) and, now and then, another
  // reference point.  It only has to keep the exponentials in range, so it moves when some row's maximum grew by more than
  // kWinSlack in the exponent.
  auto settle = [&](floatx16& nxt, int half) __attribute__((always_inline)) {
    const int v0 = 32 * half;
    if (half >= tail_half || (half < clear_half && half >= seen_sinks)) {
      const int at = v0 + 4 * hl, sinks = in.sinks - at, last = top - at, from = last - in.window + 1;
      most = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int v = (r >> 2) * 8 + (r & 3);
        const bool hidden = (v > last) | ((v < from) & (v >= sinks));
        nxt[r] = hidden ? -INFINITY : nxt[r];
        most = fmaxf(most, nxt[r]);
      }
    }
    const float mb = lane_op<32>(most, MaxOp()) * a.scale_log2e;
    if (__builtin_amdgcn_ballot_w64(mb > mb_run + kWinSlack) != 0) {
      const float mb_new = fmaxf(mb_run, mb);
      const float alpha = __builtin_amdgcn_exp2f(mb_run - mb_new);
      l_run *= alpha;
      mb_run = mb_new;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[d][r] *= alpha;
    }
  };
  // In an iteration a half's probabilities meet V while the scores of the half behind it are made, twice: so it reads halves
  // 2 i and 2 i + 1 of V and 2 i + 1 and 2 i + 2 of K, and K's tiles lie half a tile behind V's.  Both land in the iteration
  // before.  A barrier each.
  floatx16 even, odd;
  request(-32, of_k, k_lds1);
  request(0, of_v, v_lds0);
  request(32, of_k, k_lds0);
  wait_all_but<0>();
  lds_barrier();
  const floatx16 none = {-INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY,
                         -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY};
  // Half `half` from scores to output, and the scores of the next; where the wave's rows see neither, the next are scores of
  // nothing.  (Behind the last half they are of what the buffer holds, and all are masked.)
  auto advance = [&](floatx16& cur, floatx16& nxt, int half, const uint16_t* k_buf, int k_from, uint16_t* v_buf,
                     int v_from) __attribute__((always_inline)) {
    if (half < sink_halves || (half + 1 >= from_half && half < upto_half)) {
      step(cur, nxt, k_buf, k_from, v_buf, v_from);
      settle(nxt, half + 1);
    } else {
      nxt = none;
    }
  };
  {
    bf16x8 op[DSTEPS];
#pragma unroll
    for (int st = 0; st < DSTEPS; ++st) op[st] = read_k(k_lds1, 32, st);
    __builtin_amdgcn_sched_barrier(0);
    even = zero;
#pragma unroll
    for (int st = 0; st < DSTEPS; ++st) even = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[st], qf[st], even, 0, 0, 0);
    most = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) most = fmaxf(most, even[r]);
  }
  settle(even, 0);
  lds_barrier();  // (the first iteration's loads land where these scores' keys were)
  auto one_tile = [&](int half, uint16_t* k_now, uint16_t* k_then, uint16_t* v_now, uint16_t* v_then) __attribute__((always_inline)) {
    request(32 * half + 96, of_k, k_then);
    request(32 * half + 64, of_v, v_then);
    advance(even, odd, half, k_now, 0, v_now, 0);
    advance(odd, even, half + 1, k_now, 32, v_now, 32);
    wait_all_but<0>();
    lds_barrier();
  };
  for (int half = 0;; half += 4) {
    one_tile(half, k_lds0, k_lds1, v_lds0, v_lds1);
    if (half + 2 >= n_halves) break;
    one_tile(half + 2, k_lds1, k_lds0, v_lds1, v_lds0);
    if (half + 4 >= n_halves) break;
  }
  if (idle) return;

  // ---- the quotient; lane holds O[row][32 d + 8 g + 4 hl + i] ----
  const float l = lane_op<32>(l_run, AddOp());
  const float inv = l == 0.f ? 0.f : 1.f / l;  // (every score below fp32's range: 0)
  u32x2 out[DT][4];
  float check = 0.f;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {  // (a bit cast of a vector's element would be one of its first)
        const uint32_t w = pack_bf16(oacc[d][4 * g + 2 * i] * inv, oacc[d][4 * g + 2 * i + 1] * inv);
        out[d][g][i] = w;
        check = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), ones, check, false);
      }
    }
  // A hidden key's V that is not finite has made NaN of the rows that share its tile (0 times it), one that is seen NaN or an
  // infinity, by the size of its probability; and scores so far from 0 that the reference point is not their maximum's exponent
  // to a sixteenth may have left the exponential's range.  Where a row of the wave is such a one, all its rows are done again,
  // slowly.
  if (__builtin_amdgcn_ballot_w64(query < len && (!(fabsf(check) < INFINITY) || fabsf(mb_run) > 0x1p20f)) != 0) {
    float m = kLowestScore, sum = 0.f;
    floatx16 acc[DT], odd_ones[DT];  // of V's finite numbers by P; how many others a row sees
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = odd_ones[d] = zero;
    auto row_of = [&](int v) __attribute__((always_inline)) {
      v = min(v, total - 1);
      return (size_t)(v >= first ? v - first + band : v);
    };
#pragma unroll 1
    for (int v0 = 0; v0 < total; v0 += 32) {
      floatx16 z = zero;
#pragma unroll
      for (int st = 0; st < DSTEPS; ++st)
        z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16(ld16(kbase + row_of(v0 + lq) * in.k_stride + st * 16 + hl * 8)), qf[st], z, 0, 0, 0);
      float most_now = -INFINITY;
      u32x4 see[2];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int v = v0 + (r >> 2) * 8 + hl * 4 + (r & 3);
        const bool seen = (v <= top) & ((v > top - in.window) | (v < in.sinks));
        z[r] = seen ? z[r] * a.scale_log2e : -INFINITY;
        most_now = fmaxf(most_now, z[r]);
        const uint32_t one = seen ? 0x3f80u << (16 * (r & 1)) : 0u;
        see[r / 8][r % 8 / 2] = r & 1 ? see[r / 8][r % 8 / 2] | one : one;
      }
      const float m_new = fmaxf(m, lane_op<32>(most_now, MaxOp())), alpha = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      sum *= alpha;
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[d] *= alpha;
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = __builtin_amdgcn_exp2f(z[r] - m);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        u32x4 pw;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t w = pack_bf16(z[8 * x + 2 * j], z[8 * x + 2 * j + 1]);
          sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), ones, sum, false);
          pw[j] = w;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          u32x4 fine{0, 0, 0, 0}, others{0, 0, 0, 0};
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t w = vbase[row_of(v0 + 16 * x + 8 * (e / 4) + 4 * hl + e % 4) * in.v_stride + 32 * d + lq];
            const bool finite = (w & 0x7f80u) != 0x7f80u;
            fine[e / 2] |= (finite ? w : 0u) << (16 * (e & 1));
            others[e / 2] |= (finite ? 0u : 0x3f80u) << (16 * (e & 1));
          }
          acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16(fine), as_bf16(pw), acc[d], 0, 0, 0);
          odd_ones[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16(others), as_bf16(see[x]), odd_ones[d], 0, 0, 0);
        }
      }
    }
    sum = lane_op<32>(sum, AddOp());
    const float over = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = odd_ones[d][4 * g + i] > 0.f ? __uint_as_float(0x7fc00000u) : acc[d][4 * g + i] * over;
        out[d][g] = u32x2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
      }
  }
  // By way of LDS, where a wave's rows take the place of keys that all waves are done with (chunk c of row r at c ^ a swizzle), so
  // that a store writes whole rows; 8 bytes of each of 32 rows at a time, the stores took a workgroup 2 us.
  uint16_t* mine = (wave & 2 ? v_lds0 : k_lds0) + (wave & 1) * kWinRows * HD;
  auto swizzle = [](int row) { return CPR == 16 ? row & 15 : (row >> 1) & 7; };
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) *reinterpret_cast<u32x2*>(mine + lq * HD + ((4 * d + g) ^ swizzle(lq)) * 8 + 4 * hl) = out[d][g];
  __builtin_amdgcn_wave_barrier();  // (a wave's LDS accesses keep their order; the compiler has to keep it too)
#pragma unroll
  for (int j = 0; j < kWinRows / RPL; ++j) {
    const int row = j * RPL + ld_sub, at = wave_q + (row >> a.pack_log2), head = (kv * n_sub + sub) * pack + (row & (pack - 1));
    const u32x4 w = ld16(mine + row * HD + (ld_c ^ swizzle(row)) * 8);
    if (at < len) st16(in.o + (((size_t)start + at) * in.n_heads + head) * HD + ld_c * 8, w);
  }
}

// Heads of a query that a row block has together: the largest power of two that divides the group, up to 32.
static int pack_log2_of(int kv_group) {
  int p = 0;
  while (p < 5 && kv_group % (2 << p) == 0) ++p;
  return p;
}

struct WindowPlan {
  int pack_log2;
  long places, blocks;
};
static WindowPlan window_plan(const WindowRows& r) {
  WindowPlan p;
  p.pack_log2 = pack_log2_of(r.n_heads / r.n_kv_heads);
  p.places = (long)r.t / ((kWinRows * kWinWaves) >> p.pack_log2) + r.B;
  p.blocks = p.places * (r.n_heads >> p.pack_log2);
  return p;
}
bool window_attention_fits(const WindowRows& r) { return window_plan(r).blocks <= 0x7fffffffL / 256 - 8; }

hipError_t launch_window_attention(const WindowRows& r, int head_dim, hipStream_t stream) {
  if (!window_attention_fits(r)) return hipErrorInvalidValue;
  const WindowPlan p = window_plan(r);
  WindowArgs a{};
  a.r = r;
  // (no sequence is longer: sums of them and of positions stay in 32 bits)
  a.r.window = std::min(r.window, r.max_seqlen);
  a.r.sinks = std::min(r.sinks, r.max_seqlen);
  a.kv_group = r.n_heads / r.n_kv_heads;
  a.pack_log2 = p.pack_log2;
  a.places = (int)p.places;
  a.blocks = (int)p.blocks;
  a.per_xcd = (int)((p.blocks + 7) / 8);
  a.scale_log2e = 1.4426950408889634f / sqrtf((float)head_dim);
  const dim3 grid((unsigned)(8 * a.per_xcd)), threads(64 * kWinWaves);
  if (head_dim == 128) {
    hipLaunchKernelGGL(window_attention_kernel<128>, grid, threads, 0, stream, a);
    return hipGetLastError();
  }
  if (head_dim == 64) {
    hipLaunchKernelGGL(window_attention_kernel<64>, grid, threads, 0, stream, a);
    return hipGetLastError();
  }
  return hipErrorInvalidValue;
}

}  // namespace ds
