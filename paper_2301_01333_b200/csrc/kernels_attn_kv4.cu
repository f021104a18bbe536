// Attention of a few new queries per sequence over the paged 4-bit cache.
//
//   o[col] = sum_t p(t, col) V[t] / sum_t p(t, col),   p = 2^(c (q[col] . K[t]) - m[col]),   K, V = lo + code * scale
//
// A column is one (query, query head) of those that share a key/value head.  The floor is the cache read once; a key
// element is half a byte, so the work per byte is what has to be kept small: at the copy bandwidth of the whole GPU an SM
// has 2.8 lane-instructions per element of K or V, 1.4 of them on the integer / logic pipe.
//
//   * The codes go into the matrix instruction as they are: masked out of their word, nothing else.  A small whole number N
//     in the low bits of a 16-bit float is the subnormal N * 2^-24 (fp16) or N * 2^-133 (bf16), and goes on being N times that
//     past the first exponent bit, which the smallest normal numbers share their spacing with: bits 0..3 and 4..7 of a half
//     are code and 16 code of that unit, in fp16 (linear below 2^11) and in bf16 (below 2^8).  One logic instruction makes two
//     operand elements.  Scales and offsets are applied to sums, never to elements:
//       q . K[t]            = scale_t * sum_i q_i code_i + lo_t * sum_i q_i          per group
//       sum_t p_t V[t][d]   = sum_t p'_t code_td + sum_t p_t (lo_t + 7.5 scale_t) - 7.5 sum_t p'_t,   p'_t = bf16(p_t scale_t)
//     The first sum of each line is the MMA's (fp32 accumulators), and so is the last of the second (a product with ones);
//     the others are a few fp32 operations per (token, column).  p' is the only rounding before the output's; what it rounds
//     is the distance from the middle of the group's range (code - 7.5), half of what the distance from lo would lose.
//   * Keys are fp16 operands.  q, bf16, becomes fp16 exactly after its row is scaled by a power of two to at most 2^15, and by
//     2^11 where it meets 16 code (elements below 2^-25 of the largest keep an absolute 2^-36 of it).  Weights p' need
//     bf16's range: p carries a factor of 2^64, which the sum of p has as well, so that the products stay normal in fp32 for
//     weights down to 2^-57, and sums of a million of them finite for values up to 2^32.
//   * m16n8k16 MMAs with the codes as the 16-row operand: tokens are the rows of the first product and the reduction of the
//     second, so a lane's nibbles are always neighbours in memory (head-dimension neighbours; the order inside a reduction
//     axis is free, Q and P are permuted to match), and 8 columns cost 8, not 16.
//   * A warp is on its own: it takes every fourth 32-token tile of its CTA's range, copies tiles ahead into its own ring in
//     shared memory with 16-byte asynchronous copies, and keeps running maximum, sum and output of its columns in
//     registers.  No barrier until the end, where the warps of a CTA are joined in shared memory.
//   * One wave of CTAs that share all the work out equally: the 128-token blocks of every (sequence, head, chunk of columns)
//     stand in one row, of which each CTA takes an equal stretch, however unlike the lengths are.  Where a stretch ends
//     inside a sequence, the pieces are joined by a second small kernel in their order.  (Against one CTA per 2048 tokens
//     of a sequence: with equal costs for unlike pieces 97 us, so 88 for 64 ragged sequences up to 8192 tokens.)
//   * Many short sequences: a warp per (sequence, head, chunk of columns), which writes its rows itself (gc_serving.cu says when).
//   * The running maximum is a reference that is only raised when a score exceeds it by 2^8: one vote per tile instead
//     of a reduction, and the sums stay far inside fp32.
//   * The sizes of the values (one running maximum) and of the reference, when it is raised, are watched: sums of values above 2^32
//     and weights of scores above 2^26 could leave fp32, which is recorded in the status word.  1.5 us of 76 on the batch below.
// Measured: 64 ragged sequences up to 8192 tokens, 8 heads of 128, groups of 64 (323 MB): 78 us = 4.1 TB/s; without any arithmetic
// the same copies take 62, so the rest is instructions that the copies of 12 warps do not cover (about 620 a tile and eight columns,
// half of them on the integer / logic pipe).  One sequence of 131071 tokens, 32 columns (142 MB, read twice, the second time from
// the L2): 86 us, bound by instructions; its products alone, 8 clocks each on a scheduler, are 33.
#include <cuda_fp16.h>

#include <type_traits>

#include "ptx.cuh"
#include "serving.cuh"

namespace gc {

namespace {
constexpr int AK_WARPS = 4;
constexpr int AK_THREADS = AK_WARPS * 32;
constexpr int AK_TILE = 32;                  // tokens per tile of a warp
constexpr int AK_STAGES = 3;
constexpr int AK_START = 2;
constexpr float AK_RAISE = 8.0f;             // binades a score may exceed the reference by
constexpr float AK_LARGEST = 0x1p32f;        // middle or scale of a group of values, above which sums could leave fp32

template <int D, int G>
struct KvLayout {
  static constexpr int NG = D / G;
  static constexpr int ROW = D / 2;                             // bytes of codes per token
  static constexpr int PITCH = D == 64 ? 32 : 64;               // the same in shared memory
  static constexpr int CODES = AK_TILE * PITCH, PARAMS = AK_TILE * NG * 4;
  static constexpr int STAGE = 2 * (CODES + PARAMS);
  static constexpr int RING = AK_STAGES * STAGE;
};

__device__ __forceinline__ float ak_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Addresses are a register plus a constant: an addition per access would go to the pipe that unpacks the codes.
template <int DST, int SRC>
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0 + %2], [%1 + %3], 16;" ::"r"(dst), "l"(src), "n"(DST), "n"(SRC) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <int OFF>
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1 + %2];" : "=r"(v) : "r"(a), "n"(OFF));
  return v;
}
template <int OFF>
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1 + %2];" : "=h"(v) : "r"(a), "n"(OFF));
  return v;
}
template <int OFF>
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2 + %3];" : "=r"(v.x), "=r"(v.y) : "r"(a), "n"(OFF));
  return v;
}
// f(constant 0), f(constant 1), ... : loops whose index has to be one
template <int N, typename F, int I = 0>
__device__ __forceinline__ void each(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    each<N, F, I + 1>(static_cast<F&&>(f));
  }
}
// the low and the high nibbles of a word's even bytes: code and 16 code in units of the smallest 16-bit float
__device__ __forceinline__ uint32_t nib_lo(uint32_t w) { return w & 0x000f000fu; }
__device__ __forceinline__ uint32_t nib_hi(uint32_t w) { return w & 0x00f000f0u; }
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ak_max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&b);
}
__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// CTAs per SM the registers are cut for: 168 for one group of columns, 255 for two (168 at width 64).  Not everything fits: two
// groups with scales for every 32 elements spill up to 144 bytes a thread.  (More CTAs with fewer
// registers were slower: at 128 the products of a tile can no longer be kept apart, 87 against 78 us for 64 ragged sequences.)
constexpr int ak_blocks(int D, int G, int NT) { return NT == 1 ? 3 : D == 64 ? 3 : 2; }
// First of the eight elements of a row that word w of lane tg holds, KP words at a time per lane.
template <int KP>
__device__ __forceinline__ int key_elem(int w, int tg) {
  return (w / KP) * (32 * KP) + tg * (8 * KP) + (w % KP) * 8;
}
// Byte offset of 16-byte chunk c of token row r in a codes tile.  The exclusive-or spreads the rows that one load
// instruction touches over all banks: eight rows with the same chunk (keys, 4 bytes a lane), rows 0, 4, 1, 5 and 2, 6, 3, 7 with
// two neighbouring chunks (keys, 8 bytes a lane), rows 0..3, 4..7, ... with two neighbouring chunks (values).
template <int D>
__device__ __forceinline__ uint32_t code_off(int r, int c) {
  if constexpr (D == 64) return r * 32 + ((c ^ ((r >> 2) & 1)) << 4);
  const int k = (r >> 1) & 3;
  return r * 64 + ((c ^ (((k & 1) << 1) ^ ((k >> 1) * 3))) << 4);
}
}  // namespace

// The row of blocks: a sequence has one block per p.block tokens, at least one, times heads and chunks of columns.  A piece of
// work costs its blocks and a start (positions, page numbers, queries, joining the warps) worth about AK_START blocks: the row
// has that many empty ones ahead of every sequence's own, so that stretches of many short sequences are no longer than others.
__device__ __forceinline__ int length_of(const Kv4AttnParams& p, int b) {
  const int len = p.lengths[b];
  return len < 0 ? 0 : min(len, p.max_len);
}
__device__ __forceinline__ int blocks_of(const Kv4AttnParams& p, int len) { return max((len + p.block - 1) / p.block, 1) + AK_START; }
// Blocks of all sequences; called by whole warps.
__device__ __forceinline__ int64_t all_blocks(const Kv4AttnParams& p) {
  int64_t all = 0;
  for (int s = threadIdx.x & 31; s < p.B; s += 32) all += blocks_of(p, length_of(p, s));
#pragma unroll
  for (int d = 16; d; d >>= 1) all += __shfl_xor_sync(0xffffffffu, all, d);
  return all;
}
// The sequence that has block number `at`, and the blocks before it; called by whole warps.
__device__ __forceinline__ int sequence_at(const Kv4AttnParams& p, int64_t at, int64_t* before) {
  const int lane = threadIdx.x & 31;
  int64_t base = 0;
  for (int s0 = 0; s0 < p.B; s0 += 32) {
    const int s = s0 + lane;
    int64_t incl = s < p.B ? blocks_of(p, length_of(p, s)) : 0;
    const int64_t own = incl;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    const uint32_t hit = __ballot_sync(0xffffffffu, s < p.B && base + incl > at);
    if (hit) {
      const int w = __ffs(hit) - 1;
      *before = base + __shfl_sync(0xffffffffu, incl - own, w);
      return s0 + w;
    }
    base += __shfl_sync(0xffffffffu, incl, 31);
  }
  *before = base;
  return p.B - 1;
}

// The logarithm of the sum of a column's exponentials, from its reference (in binades) and the sum relative to it, which carries
// a factor of 2^64 (taken out before the logarithm, which has a step of 2^-17 beyond 64); minus infinity where the column saw nothing.
__device__ __forceinline__ float log_of_sum(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l * 0x1p-64f)) * 0.693147180559945309f; }
__device__ __forceinline__ float* lse_of(const Kv4AttnParams& p, int b, int query, int head) {
  return p.lse + (static_cast<int64_t>(b) * p.n + query) * p.Hq + head;
}

// Blocks k0 .. k0 + kn of the nb of head hk of sequence b (len tokens), columns of one chunk.  NT: groups of eight columns.
// SOLO: this warp alone does all of it.
template <int D, int G, int NT, bool SOLO>
__device__ __forceinline__ void segment(const Kv4AttnParams& p, uint8_t* smem, int b, int hk, int chunk, int len, int k0, int kn, int nb) {
  using L = KvLayout<D, G>;
  constexpr int NG = L::NG, KW = D / 32, MT = D / 16, COLS = 8 * NT;
  constexpr int UG = G / 32;                                     // 16-bit units of V per lane, token and group
  constexpr int KP = G >= 64 ? 2 : 1;                            // words of K a lane loads at a time
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane >> 2, tg = lane & 3;
  const int columns = p.n * p.g, col0 = chunk * COLS;
  const int t_begin = k0 * p.block, t_end = min(len, (k0 + kn) * p.block);

  const int tiles = t_end > t_begin ? (t_end - t_begin + AK_TILE - 1) / AK_TILE : 0;
  const int mine = SOLO ? tiles : tiles > warp ? (tiles - warp + AK_WARPS - 1) / AK_WARPS : 0;      // tiles warp, warp + 4, ...
  auto token_of = [&](int i) { return t_begin + (SOLO ? i : warp + AK_WARPS * i) * AK_TILE; };
  const uint32_t ring_a = smem_u32(smem + warp * L::RING);
  const int* trow = p.table + b * p.table_stride;
  const int page_mask = (1 << p.page_shift) - 1;
  const bool one_page = p.page_shift >= 5;                       // a tile of 32 tokens lies in one page, else in two

  // 16-byte chunks of codes a lane copies of each half tile, and where they go
  constexpr int CH = L::ROW / 16, N = 16 * CH, IT = (N + 31) / 32, PN = NG * 4;
  uint32_t soff[IT];
#pragma unroll
  for (int k = 0; k < IT; ++k) {
    const int x = k * 32 + lane, r = x / CH;
    soff[k] = code_off<D>(r, x - r * CH);
  }
  // Page numbers of 16 tiles at a time, two per tile, one per lane.
  int pages = 0;
  auto fetch_pages = [&](int i) {
    const int tok = token_of(i + (lane >> 1)) + (lane & 1) * 16;
    pages = 0;
    if (tok < t_end) {
      pages = trow[tok >> p.page_shift];
      if (pages < 0 || pages >= p.num_pages) {
        report(p.status, DEV_BAD_PAGE);
        pages = 0;
      }
    }
  };
  const uint32_t poff = (lane & 15) * 16 + (lane < 16 ? 0 : L::PARAMS);
  const uint8_t* kbase = p.k_codes + lane * 16;
  const int64_t to_v = p.v_codes - p.k_codes;
  const uint8_t* pbase = reinterpret_cast<const uint8_t*>(lane < 16 ? p.k_params : p.v_params) + (lane & 15) * 16;
  // half H of the tile at shared address st, of which the first half would be row `row` of the cache
  auto copy_half = [&](auto half_c, uint32_t st, const uint8_t* ks, const uint8_t* vs, const uint8_t* ps) {
    constexpr int H = decltype(half_c)::value, TO = H * 16 * L::PITCH, FROM = H * 16 * L::ROW, PB = H * 16 * NG * 4;
    each<IT>([&](auto k) {
      if (N % 32 == 0 || k * 32 + lane < N) {
        cp_async16<TO, FROM + k * 512>(st + soff[k], ks);
        cp_async16<TO + L::CODES, FROM + k * 512>(st + soff[k], vs);
      }
    });
    if ((lane & 15) < PN) cp_async16<2 * L::CODES + PB, PB>(st + poff, ps);
  };
  uint32_t st_in = ring_a;                                       // the stage the next copy goes to
  auto issue = [&](int i) {
    if (i < mine) {
      if ((i & 15) == 0) fetch_pages(i);
      const int t0 = token_of(i);
      const int64_t row = ((static_cast<int64_t>(__shfl_sync(0xffffffffu, pages, 2 * (i & 15))) * p.Hk + hk) << p.page_shift) + (t0 & page_mask);
      const uint8_t* ks = kbase + row * L::ROW;
      const uint8_t* ps = pbase + row * (NG * 4);
      copy_half(std::integral_constant<int, 0>{}, st_in, ks, ks + to_v, ps);
      if (t0 + 16 < t_end) {
        if (!one_page) {                                         // the second half's rows, 16 of them back
          const int64_t row1 = ((static_cast<int64_t>(__shfl_sync(0xffffffffu, pages, 2 * (i & 15) + 1)) * p.Hk + hk) << p.page_shift) - 16;
          ks = kbase + row1 * L::ROW;
          ps = pbase + row1 * (NG * 4);
        }
        copy_half(std::integral_constant<int, 1>{}, st_in, ks, ks + to_v, ps);
      }
    }
    cp_commit();
    st_in += L::STAGE;
    if (st_in == ring_a + L::RING) st_in = ring_a;
  };

#pragma unroll
  for (int i = 0; i < AK_STAGES - 1; ++i) issue(i);              // under way while the queries are prepared

  // Queries as the second operand of the first product: lane (gr, tg) holds of column gr, of every 32 KP elements, the
  // eight (or sixteen, where a group spans 64) that its lane of the first operand holds: element 8 x + y of the lane's run
  // in the order (0,4), (1,5), (2,6), (3,7) in which the nibbles of a word come apart.
  uint32_t qf[NT][KW][4];
  float sq[NT][NG][2];                                           // sum of q over a group, columns 2 tg and 2 tg + 1
  float ce[NT][2];                                               // c times the power of two the scores are short of
  int lim[NT][2];                                                // tokens that column sees
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int col = col0 + nt * 8 + gr;
    const bool ok = col < columns;
    const int qi = ok ? col / p.g : 0, hh = ok ? col - qi * p.g : 0;
    const __nv_bfloat16* qrow = p.q + b * p.qb + qi * p.qn + static_cast<int64_t>(hk * p.g + hh) * p.qh;
    uint4 v[KW];
    float top = 0.f;
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      v[w] = make_uint4(0, 0, 0, 0);
      if (ok) v[w] = *reinterpret_cast<const uint4*>(qrow + key_elem<KP>(w, tg));
      const uint32_t x[4] = {v[w].x, v[w].y, v[w].z, v[w].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(bf_lo(x[i])), fabsf(bf_hi(x[i]))));
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // 2^e > top >= 2^(e - 1): q / 2^e lies in (-1, 1).  (Rows of zeros and of infinities: e = 0; subnormal tops: the smallest e.)
    const int ex = static_cast<int>(__float_as_uint(top) >> 23);
    const int e = top == 0.f || ex == 255 ? 0 : max(ex, 1) - 126;
    const float down = __uint_as_float(static_cast<uint32_t>(127 - e / 2) << 23), down2 = __uint_as_float(static_cast<uint32_t>(127 - (e - e / 2)) << 23);
    float ss[NG];
#pragma unroll
    for (int j = 0; j < NG; ++j) ss[j] = 0.f;
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      const uint32_t x[4] = {v[w].x, v[w].y, v[w].z, v[w].w};
      float y[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[2 * i] = bf_lo(x[i]) * down * down2;
        y[2 * i + 1] = bf_hi(x[i]) * down * down2;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float f = i & 1 ? 0x1p11f : 0x1p15f;               // the odd ones meet 16 code
        const __half2 h = __floats2half2_rn(y[i] * f, y[i + 4] * f);
        qf[nt][w][i] = *reinterpret_cast<const uint32_t*>(&h);
        ss[w * 32 / G] += (__low2float(h) + __high2float(h)) * (0x1p-9f / f);      // in the unit of the product: 2^(15 - 24)
      }
    }
#pragma unroll
    for (int j = 0; j < NG; ++j) {
#pragma unroll
      for (int d = 1; d < 4; d <<= 1) ss[j] += __shfl_xor_sync(0xffffffffu, ss[j], d);
#pragma unroll
      for (int i = 0; i < 2; ++i) sq[nt][j][i] = __shfl_sync(0xffffffffu, ss[j], 8 * tg + 4 * i);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int cc = col0 + nt * 8 + 2 * tg + i;
      lim[nt][i] = cc < columns ? len - (p.n - 1) + cc / p.g : 0;
      const int ee = __shfl_sync(0xffffffffu, e, 8 * tg + 4 * i);
      ce[nt][i] = p.c * 0x1p9f * __uint_as_float(static_cast<uint32_t>(127 + ee / 2) << 23) * __uint_as_float(static_cast<uint32_t>(127 + ee - ee / 2) << 23);
    }
  }

  float o[NT][MT][4], mneg[NT][2], thr[NT][2], l[NT][2], z[NT][NG][2], ws[NT][NG][4];
  float largest = 0.f;                                           // middle or scale of the values seen (NaN apart)
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int i = 0; i < MT; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
#pragma unroll
    for (int j = 0; j < NG; ++j) ws[nt][j][0] = ws[nt][j][1] = ws[nt][j][2] = ws[nt][j][3] = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      mneg[nt][i] = INFINITY;                                    // 64 minus the reference, in binades; none yet
      thr[nt][i] = -INFINITY;                                    // the score (before ce) from which it has to be raised
      l[nt][i] = 0.f;
#pragma unroll
      for (int j = 0; j < NG; ++j) z[nt][j][i] = 0.f;
    }
  }

  // Row r of a 16-row operand is token perm(r) = r / 2 (r even), 4 + r / 2 (r odd), + 8 above
  const int pr = (gr >> 1) + ((gr & 1) << 2);
  uint32_t koff[KW / KP], voff[NG][2];                           // where a lane's codes lie in the first rows of a tile
#pragma unroll
  for (int w = 0; w < KW / KP; ++w) koff[w] = code_off<D>(pr, (w * KP * 16 + tg * KP * 4) >> 4) + ((w * KP * 16 + tg * KP * 4) & 15);
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    const int byte = j * (G / 2) + gr * (G / 16);
    voff[j][0] = code_off<D>(tg, byte >> 4) + (byte & 15);
    voff[j][1] = code_off<D>(tg + 4, byte >> 4) + (byte & 15);   // rows 4 and 12 apart have another key, rows 8 and 16 apart the same
  }
  // One tile: scores, reference, probabilities, second product.  EDGE: some column may not see all of it (the columns'
  // limits lie within n of the sequence's end; padding columns see nothing and are left as they come: nobody reads them).
  auto tile = [&](auto edge_c, int i, uint32_t kc) {
    constexpr bool EDGE = decltype(edge_c)::value;
    const int t0 = token_of(i);
    const uint32_t kp = kc + pr * NG * 4;
    float s[2][NT][4];
    // Sums of one (16 rows, group) depend on one another: where registers allow, those of all groups take turns, else those
    // of the two row blocks.
    constexpr int JI = NG <= 2 ? NG : NT > 1 ? 1 : NG == 3 ? 3 : 2;            // groups in turn
    each<NG / JI>([&](auto jo_c) {
      float acc[JI][2][NT][4];
#pragma unroll
      for (int j = 0; j < JI; ++j)
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) acc[j][mt][nt][0] = acc[j][mt][nt][1] = acc[j][mt][nt][2] = acc[j][mt][nt][3] = 0.f;
      each<G / 32 / KP>([&](auto w_c) {
        uint32_t raw[JI][2][2][KP];                              // words of rows gr and gr + 8
        each<JI>([&](auto ji_c) {
          each<2>([&](auto mt_c) {
            constexpr int ji = decltype(ji_c)::value, mt = decltype(mt_c)::value;
            constexpr int w0 = (decltype(jo_c)::value * JI + ji) * (G / 32) + decltype(w_c)::value * KP;
            const uint32_t aa = kc + koff[w0 / KP];              // 8 rows further down: the same key
            constexpr int ra = mt * 16 * L::PITCH, rb = ra + 8 * L::PITCH;
            if constexpr (KP == 2) {
              const uint2 x = lds64<ra>(aa), y = lds64<rb>(aa);
              raw[ji][mt][0][0] = x.x; raw[ji][mt][0][1] = x.y;
              raw[ji][mt][1][0] = y.x; raw[ji][mt][1][1] = y.y;
            } else {
              raw[ji][mt][0][0] = lds32<ra>(aa);
              raw[ji][mt][1][0] = lds32<rb>(aa);
            }
          });
        });
#pragma unroll
        for (int x = 0; x < KP; ++x) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {                 // neighbouring products belong to different sums
#pragma unroll
            for (int ji = 0; ji < JI; ++ji) {
#pragma unroll
              for (int mt = 0; mt < 2; ++mt) {
                const int w = (decltype(jo_c)::value * JI + ji) * (G / 32) + decltype(w_c)::value * KP + x;
                const uint32_t ka = half ? raw[ji][mt][0][x] >> 8 : raw[ji][mt][0][x], kb = half ? raw[ji][mt][1][x] >> 8 : raw[ji][mt][1][x];
                const uint32_t a0 = nib_lo(ka), a1 = nib_lo(kb), a2 = nib_hi(ka), a3 = nib_hi(kb);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_f16(acc[ji][mt][nt], a0, a1, a2, a3, qf[nt][w][2 * half], qf[nt][w][2 * half + 1]);
              }
            }
          }
        }
      });
      each<JI>([&](auto ji_c) {
        each<2>([&](auto mt_c) {
          constexpr int ji = decltype(ji_c)::value, mt = decltype(mt_c)::value, j = decltype(jo_c)::value * JI + ji;
          constexpr int po = 2 * L::CODES + (mt * 16 * NG + j) * 4;
          const uint32_t pa = lds32<po>(kp), pb = lds32<po + 8 * NG * 4>(kp);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const float* ac = acc[ji][mt][nt];
            float* sc = s[mt][nt];
            if (j == 0) {
              sc[0] = fmaf(bf_hi(pa), ac[0], bf_lo(pa) * sq[nt][j][0]);
              sc[1] = fmaf(bf_hi(pa), ac[1], bf_lo(pa) * sq[nt][j][1]);
              sc[2] = fmaf(bf_hi(pb), ac[2], bf_lo(pb) * sq[nt][j][0]);
              sc[3] = fmaf(bf_hi(pb), ac[3], bf_lo(pb) * sq[nt][j][1]);
            } else {
              sc[0] = fmaf(bf_hi(pa), ac[0], fmaf(bf_lo(pa), sq[nt][j][0], sc[0]));
              sc[1] = fmaf(bf_hi(pa), ac[1], fmaf(bf_lo(pa), sq[nt][j][1], sc[1]));
              sc[2] = fmaf(bf_hi(pb), ac[2], fmaf(bf_lo(pb), sq[nt][j][0], sc[2]));
              sc[3] = fmaf(bf_hi(pb), ac[3], fmaf(bf_lo(pb), sq[nt][j][1], sc[3]));
            }
          }
        });
      });
    });
    if constexpr (EDGE) {
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        const int ta = t0 + mt * 16 + pr;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int t = ta + (e >> 1) * 8;
            if (t >= lim[nt][e & 1] || t >= t_end) s[mt][nt][e] = -INFINITY;
          }
        }
      }
    }
    // ---- the reference of the exponentials
    bool over = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
        over |= fmaxf(fmaxf(s[0][nt][e], s[0][nt][e + 2]), fmaxf(s[1][nt][e], s[1][nt][e + 2])) > thr[nt][e];
    }
    if (__any_sync(0xffffffffu, over)) {
      bool too_large = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float mx = fmaxf(fmaxf(s[0][nt][e], s[0][nt][e + 2]), fmaxf(s[1][nt][e], s[1][nt][e + 2]));
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
          const float mo = 64.f - mneg[nt][e], mn = fmaxf(mo, mx * ce[nt][e]);
          const float f = mo == mn ? 1.f : ak_ex2(mo - mn);      // 0 from the initial minus infinity
          if (mo != mn) {
            too_large |= score_too_large(mn);
            mneg[nt][e] = 64.f - mn;
            thr[nt][e] = mx + AK_RAISE / ce[nt][e];
          }
          l[nt][e] *= f;
#pragma unroll
          for (int j = 0; j < NG; ++j) {
            z[nt][j][e] *= f;
            ws[nt][j][e] *= f;
            ws[nt][j][e + 2] *= f;
          }
#pragma unroll
          for (int k = 0; k < MT; ++k) {
            o[nt][k][e] *= f;
            o[nt][k][e + 2] *= f;
          }
        }
      }
      if (too_large) report(p.status, DEV_LARGE_SCORE);
    }
    // ---- probabilities and the second product, 16 tokens at a time
    each<2>([&](auto mt_c) {
      constexpr int mt = decltype(mt_c)::value;
      float pw[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        pw[nt][0] = ak_ex2(fmaf(s[mt][nt][0], ce[nt][0], mneg[nt][0]));
        pw[nt][1] = ak_ex2(fmaf(s[mt][nt][1], ce[nt][1], mneg[nt][1]));
        pw[nt][2] = ak_ex2(fmaf(s[mt][nt][2], ce[nt][0], mneg[nt][0]));
        pw[nt][3] = ak_ex2(fmaf(s[mt][nt][3], ce[nt][1], mneg[nt][1]));
        if constexpr (EDGE) {                                    // (a column that has seen nothing yet has no reference)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (s[mt][nt][e] == -INFINITY) pw[nt][e] = 0.f;
        }
        l[nt][0] += pw[nt][0] + pw[nt][2];
        l[nt][1] += pw[nt][1] + pw[nt][3];
      }
      each<NG>([&](auto j_c) {
        constexpr int j = decltype(j_c)::value;
        constexpr int po = 2 * L::CODES + L::PARAMS + (mt * 16 * NG + j) * 4;
        const uint32_t pa = lds32<po>(kp), pb = lds32<po + 8 * NG * 4>(kp);
        const float sa = bf_hi(pa), sb = bf_hi(pb);
        const float ma = fmaf(7.5f, sa, bf_lo(pa)), mb = fmaf(7.5f, sb, bf_lo(pb));     // the middle of a group's range
        if constexpr (EDGE) {
          const int ta = t0 + mt * 16 + pr;
          if (ta < t_end) largest = ak_max3(largest, sa, fabsf(ma));
          if (ta + 8 < t_end) largest = ak_max3(largest, sb, fabsf(mb));
        } else {
          largest = ak_max3(largest, sa, sb);
          largest = ak_max3(largest, fabsf(ma), fabsf(mb));
        }
        uint32_t bf[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float x0 = pw[nt][0] * sa, x1 = pw[nt][1] * sa, x2 = pw[nt][2] * sb, x3 = pw[nt][3] * sb;
          if constexpr (EDGE) {                                  // a weight of zero hides whatever the cache holds there
            const bool h0 = s[mt][nt][0] == -INFINITY, h1 = s[mt][nt][1] == -INFINITY, h2 = s[mt][nt][2] == -INFINITY, h3 = s[mt][nt][3] == -INFINITY;
            x0 = h0 ? 0.f : x0;
            x1 = h1 ? 0.f : x1;
            x2 = h2 ? 0.f : x2;
            x3 = h3 ? 0.f : x3;
            z[nt][j][0] += (h0 ? 0.f : pw[nt][0] * ma) + (h2 ? 0.f : pw[nt][2] * mb);
            z[nt][j][1] += (h1 ? 0.f : pw[nt][1] * ma) + (h3 ? 0.f : pw[nt][3] * mb);
          } else {
            z[nt][j][0] = fmaf(pw[nt][0], ma, fmaf(pw[nt][2], mb, z[nt][j][0]));
            z[nt][j][1] = fmaf(pw[nt][1], ma, fmaf(pw[nt][3], mb, z[nt][j][1]));
          }
          bf[nt][0] = transpose8x8(pack_bf16(x0, x1));
          bf[nt][1] = transpose8x8(pack_bf16(x2, x3));
          mma_bf16(ws[nt][j], 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, bf[nt][0], bf[nt][1]);
        }
        // lane (gr, tg): tokens tg, tg + 4, tg + 8, tg + 12 of the 16; elements j G + gr G / 8 + 2 byte + nibble
        uint32_t vw[4][(UG + 1) / 2];
        each<4>([&](auto k) {
          const uint32_t a = kc + voff[j][k & 1];
          constexpr int ro = L::CODES + (mt * 16 + (k & 2) * 4) * L::PITCH;
          if constexpr (UG == 1) vw[k][0] = lds16<ro>(a);
          if constexpr (UG == 2) vw[k][0] = lds32<ro>(a);
          if constexpr (UG == 4) {
            const uint2 t = lds64<ro>(a);
            vw[k][0] = t.x;
            vw[k][1] = t.y;
          }
        });
#pragma unroll
        for (int u = 0; u < 2 * UG; ++u) {
          // byte u of the lane's run, of tokens (0, 1) and (2, 3) of its four
          const uint32_t sel = 0x0400u | ((u & 3) * 0x1111u);
          const uint32_t x = __byte_perm(vw[0][u >> 2], vw[1][u >> 2], sel), y = __byte_perm(vw[2][u >> 2], vw[3][u >> 2], sel);
          const uint32_t a0 = nib_lo(x), a1 = nib_hi(x), a2 = nib_lo(y), a3 = nib_hi(y);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma_bf16(o[nt][j * 2 * UG + u], a0, a1, a2, a3, bf[nt][0], bf[nt][1]);
        }
      });
    });
  };

  uint32_t st_out = ring_a;                                      // the stage the next tile is read from
  for (int i = 0; i < mine; ++i) {
    cp_wait<AK_STAGES - 2>();
    __syncwarp();
    const int t_next = token_of(i) + AK_TILE;
    if (t_next > len - (p.n - 1) || t_next > t_end) tile(std::true_type{}, i, st_out);
    else tile(std::false_type{}, i, st_out);
    __syncwarp();
    issue(i + AK_STAGES - 1);
    st_out += L::STAGE;
    if (st_out == ring_a + L::RING) st_out = ring_a;
  }
  cp_wait<0>();
  if (largest > AK_LARGEST) report(p.status, DEV_LARGE_VALUE);

  // ---- join the warps: (m, l) and the outputs of every column through shared memory
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], d);
#pragma unroll
        for (int j = 0; j < NG; ++j) z[nt][j][e] += __shfl_xor_sync(0xffffffffu, z[nt][j][e], d);
      }
    }
  }
  if constexpr (SOLO) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int cc = col0 + nt * 8 + 2 * tg + e;
        if (cc >= columns) continue;
        const float r = l[nt][e] == 0.f ? 0.f : 1.0f / l[nt][e];
        const int qi = cc / p.g, hh = cc - qi * p.g;
        if (p.lse && gr == 0) *lse_of(p, b, qi, hk * p.g + hh) = log_of_sum(64.f - mneg[nt][e], l[nt][e]);
        __nv_bfloat16* dst = p.o + b * p.ob + qi * p.on + static_cast<int64_t>(hk * p.g + hh) * p.oh + gr * (G / 8);
#pragma unroll
        for (int j = 0; j < NG; ++j) {
          const float mid = fmaf(-7.5f, ws[nt][j][e], z[nt][j][e]);
#pragma unroll
          for (int u = 0; u < UG; ++u) {
            const int k = (j * UG + u) * 2;
            *reinterpret_cast<uint2*>(dst + j * G + 4 * u) =
                make_uint2(pack_bf16(fmaf(o[nt][k][e] * 0x1p67f, 0x1p66f, mid) * r, fmaf(o[nt][k][e + 2] * 0x1p67f, 0x1p62f, mid) * r),
                           pack_bf16(fmaf(o[nt][k + 1][e] * 0x1p67f, 0x1p66f, mid) * r, fmaf(o[nt][k + 1][e + 2] * 0x1p67f, 0x1p62f, mid) * r));
          }
        }
      }
    }
    return;
  }
  __syncthreads();                                               // the rings are free
  constexpr int OP = D + 4;                                      // row pitch: neighbouring columns on other banks
  float* s_o = reinterpret_cast<float*>(smem);                   // [warps][COLS][OP]
  float* s_m = s_o + AK_WARPS * COLS * OP;                       // [warps][COLS]
  float* s_l = s_m + AK_WARPS * COLS;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int col = nt * 8 + 2 * tg + e;
      float* row = s_o + (warp * COLS + col) * OP;
#pragma unroll
      for (int j = 0; j < NG; ++j) {
#pragma unroll
        for (int u = 0; u < UG; ++u) {
          const int k = (j * UG + u) * 2;
          const float mid = fmaf(-7.5f, ws[nt][j][e], z[nt][j][e]);
          *reinterpret_cast<float4*>(row + j * G + gr * (G / 8) + 4 * u) =
              make_float4(fmaf(o[nt][k][e] * 0x1p67f, 0x1p66f, mid), fmaf(o[nt][k][e + 2] * 0x1p67f, 0x1p62f, mid),
                          fmaf(o[nt][k + 1][e] * 0x1p67f, 0x1p66f, mid), fmaf(o[nt][k + 1][e + 2] * 0x1p67f, 0x1p62f, mid));
        }
      }
      if (gr == 0) {
        s_m[warp * COLS + col] = 64.f - mneg[nt][e];
        s_l[warp * COLS + col] = l[nt][e];
      }
    }
  }
  __syncthreads();
  const int cols_here = min(COLS, columns - col0);
  for (int x = threadIdx.x; x < cols_here * (D / 4); x += AK_THREADS) {
    const int col = x / (D / 4), d = (x - col * (D / 4)) * 4;
    float mm = -INFINITY;
#pragma unroll
    for (int w = 0; w < AK_WARPS; ++w) mm = fmaxf(mm, s_m[w * COLS + col]);
    // A warp in which the column saw nothing has minus infinity, and sums of zero; one whose scores are all NaN has minus infinity
    // too, but sums that are NaN, which a factor of zero lets through.
    const float ref = mm == -INFINITY ? 0.f : mm;
    float ll = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < AK_WARPS; ++w) {
      const float f = ak_ex2(s_m[w * COLS + col] - ref);
      const float4 v = *reinterpret_cast<const float4*>(s_o + (w * COLS + col) * OP + d);
      ll = fmaf(f, s_l[w * COLS + col], ll);
      a.x = fmaf(f, v.x, a.x);
      a.y = fmaf(f, v.y, a.y);
      a.z = fmaf(f, v.z, a.z);
      a.w = fmaf(f, v.w, a.w);
    }
    if (kn == nb) {
      const float r = ll == 0.f ? 0.f : 1.0f / ll;
      const int cc = col0 + col, qi = cc / p.g, hh = cc - qi * p.g;
      if (p.lse && d == 0) *lse_of(p, b, qi, hk * p.g + hh) = log_of_sum(mm, ll);
      __nv_bfloat16* dst = p.o + b * p.ob + qi * p.on + static_cast<int64_t>(hk * p.g + hh) * p.oh + d;
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(a.x * r, a.y * r), pack_bf16(a.z * r, a.w * r));
    } else {
      // a CTA has at most one piece that begins inside a sequence and one that begins with it and does not reach its end
      const int64_t piece = (2 * static_cast<int64_t>(blockIdx.x) + (k0 == 0)) * COLS + col;
      const int64_t pieces = 2 * static_cast<int64_t>(gridDim.x) * COLS;
      *reinterpret_cast<float4*>(p.ws + piece * D + d) = a;
      if (d == 0) *reinterpret_cast<float2*>(p.ws + pieces * D + piece * 2) = make_float2(mm, ll);
    }
  }
  __syncthreads();                                               // the next segment's copies may overwrite what was joined
}

// Which (sequence, head, chunk) a CTA left a piece of: one that begins with it and does not reach its end, and one that begins
// inside it; -1: none.  Behind the pieces in the workspace, one per CTA.
struct PiecesOf {
  int start, inside;
};
template <int D>
__device__ __forceinline__ PiecesOf* pieces_of(const Kv4AttnParams& p, int cols, int ctas) {
  return reinterpret_cast<PiecesOf*>(p.ws + 2 * static_cast<int64_t>(ctas) * cols * (D + 2));
}

template <int D, int G, int NT, bool SOLO>
__global__ void __launch_bounds__(AK_THREADS, ak_blocks(D, G, NT)) attn_kv4_kernel(const __grid_constant__ Kv4AttnParams p) {
  extern __shared__ uint4 smem_u4[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(smem_u4);

  wait_for_predecessor();
  const int per_seq = p.Hk * p.col_chunks;
  int b, u, len, nb, k0 = 0;                                     // sequence, (head, chunk), its length, blocks, first block of mine
  int64_t left;                                                  // blocks to do
  if constexpr (SOLO) {                                          // a warp per (sequence, head, chunk)
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * AK_WARPS + (threadIdx.x >> 5);
    if (unit >= static_cast<int64_t>(p.B) * per_seq) return;
    b = static_cast<int>(unit / per_seq);
    u = static_cast<int>(unit - static_cast<int64_t>(b) * per_seq);
    if (u == 0 && (threadIdx.x & 31) == 0 && (p.lengths[b] < 0 || p.lengths[b] > p.max_len)) report(p.status, DEV_BAD_LENGTH);
    segment<D, G, NT, true>(p, smem, b, u / p.col_chunks, u % p.col_chunks, length_of(p, b), 0, 1, 1);
    return;
  }
  if (p.block >= p.max_len) {                                    // nothing is split: a CTA per (sequence, head, chunk)
    b = blockIdx.x / per_seq;
    u = blockIdx.x - b * per_seq;
    if (u == 0 && threadIdx.x == 0 && (p.lengths[b] < 0 || p.lengths[b] > p.max_len)) report(p.status, DEV_BAD_LENGTH);
    len = length_of(p, b);
    left = nb = blocks_of(p, len);
  } else {
    // my stretch of the row of blocks, and the sequence it begins in
    const int64_t total = all_blocks(p) * per_seq;
    if (gridDim.x > 1 && threadIdx.x == 0) *(pieces_of<D>(p, 8 * NT, gridDim.x) + blockIdx.x) = {-1, -1};
    if (blockIdx.x == 0 && threadIdx.x < 32) {
      for (int s = threadIdx.x; s < p.B; s += 32)
        if (p.lengths[s] < 0 || p.lengths[s] > p.max_len) report(p.status, DEV_BAD_LENGTH);
    }
    const int64_t ctas = min(static_cast<int64_t>(gridDim.x), total);        // none is left without a block
    if (blockIdx.x >= ctas) return;
    int64_t cur = total * blockIdx.x / ctas, skipped;
    left = total * (blockIdx.x + 1) / ctas - cur;
    b = sequence_at(p, cur / per_seq, &skipped);
    cur -= skipped * per_seq;                                    // from here on relative to the sequence's first block
    len = length_of(p, b);
    nb = blocks_of(p, len);
    u = static_cast<int>(cur / nb);
    k0 = static_cast<int>(cur - static_cast<int64_t>(u) * nb);
  }
  for (; left > 0;) {
    const int kn = static_cast<int>(min(static_cast<int64_t>(nb - k0), left));
    const int first = max(k0 - AK_START, 0), behind = k0 + kn - AK_START;
    if (behind > first) {
      if (behind - first < nb - AK_START && threadIdx.x == 0) {
        PiecesOf* mine = pieces_of<D>(p, 8 * NT, gridDim.x) + blockIdx.x;
        (first == 0 ? mine->start : mine->inside) = b * per_seq + u;
      }
      segment<D, G, NT, false>(p, smem, b, u / p.col_chunks, u % p.col_chunks, len, first, behind - first, nb - AK_START);
    }
    left -= kn;
    k0 = 0;
    if (++u == per_seq && left > 0) {
      u = 0;
      len = length_of(p, ++b);
      nb = blocks_of(p, len);
    }
  }
}
// Joins the pieces of a split sequence for one column, in a fixed order.  JW = 1: a warp per column, four to a CTA.  JW = 8:
// a CTA per column, each warp every eighth piece, then the warps; for sequences in many pieces, which one warp would read one
// memory latency after the other (one sequence of 8000 tokens in 55: 27 us against 17; but 64 of them in two or three: 125
// against 136, for so many CTAs have to be started).  The choice goes by the average: one long sequence among many short ones is
// joined by one warp a column.  Which CTAs left the pieces is looked up in what they noted, so that nothing is read before the wait
// (one sequence of 8000 tokens 14.2 us; with the lengths read ahead of the wait, which nothing allows, 13.5).
template <int D, int JW>
__global__ void __launch_bounds__(JW == 1 ? 128 : JW * 32) attn_kv4_join_kernel(const __grid_constant__ Kv4AttnParams p, const int cols, const int ctas) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ float4 s_o[JW][32];
  __shared__ float s_l[JW];
  const int lane = threadIdx.x & 31, warp = JW == 1 ? 0 : threadIdx.x >> 5;
  const int columns = p.n * p.g;
  const int64_t items = static_cast<int64_t>(p.B) * p.Hk * columns;
  const int64_t item = min(JW == 1 ? static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5) : blockIdx.x, items - 1);   // (a surplus warp repeats the last)
  const int bh = static_cast<int>(item / columns), cc = static_cast<int>(item - static_cast<int64_t>(bh) * columns);
  const int b = bh / p.Hk, hk = bh - b * p.Hk, chunk = cc / cols;
  const int unit = bh * p.col_chunks + chunk;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // the CTA it begins in, and how many more have a piece of it: those that follow
  const PiecesOf* noted = pieces_of<D>(p, cols, ctas);
  int c0 = -1, n = 0;
  for (int s0 = lane; s0 < ctas; s0 += 512) {                    // (three CTAs an SM: one round of loads, all under way at once)
    int2 x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      x[i] = make_int2(-1, -1);
      if (s0 + 32 * i < ctas) x[i] = *reinterpret_cast<const int2*>(noted + s0 + 32 * i);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (x[i].x == unit) c0 = s0 + 32 * i;
      n += x[i].y == unit;
    }
  }
  c0 = __reduce_max_sync(0xffffffffu, c0);
  if (c0 < 0) return;                                            // never split: written by its CTA
  n = __reduce_add_sync(0xffffffffu, n) + 1;
  auto piece_of = [&](int s) { return (2 * static_cast<int64_t>(c0 + s) + (s == 0)) * cols + (cc - chunk * cols); };
  const float2* ml = reinterpret_cast<const float2*>(p.ws + 2 * static_cast<int64_t>(ctas) * cols * D);
  float mm = -INFINITY;
  for (int s = lane; s < n; s += 32) mm = fmaxf(mm, ml[piece_of(s)].x);
#pragma unroll
  for (int d = 16; d; d >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, d));
  float ll = 0.f;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  const bool live = lane * 4 < D;
  const float ref = mm == -INFINITY ? 0.f : mm;                  // (as where the warps are joined: NaN sums pass)
#pragma unroll 4
  for (int s = warp; s < n; s += JW) {
    const int64_t piece = piece_of(s);
    const float2 x = ml[piece];
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (live) v = *reinterpret_cast<const float4*>(p.ws + piece * D + lane * 4);
    const float f = ak_ex2(x.x - ref);                           // 0 for a piece in which this column sees nothing
    ll = fmaf(f, x.y, ll);
    a.x = fmaf(f, v.x, a.x);
    a.y = fmaf(f, v.y, a.y);
    a.z = fmaf(f, v.z, a.z);
    a.w = fmaf(f, v.w, a.w);
  }
  if constexpr (JW > 1) {
    s_o[warp][lane] = a;
    if (lane == 0) s_l[warp] = ll;
    __syncthreads();
    if (warp != 0) return;
#pragma unroll
    for (int w = 1; w < JW; ++w) {
      const float4 v = s_o[w][lane];
      a.x += v.x;
      a.y += v.y;
      a.z += v.z;
      a.w += v.w;
      ll += s_l[w];
    }
  }
  if (!live) return;
  const float r = ll == 0.f ? 0.f : 1.0f / ll;
  const int qi = cc / p.g, hh = cc - qi * p.g;
  if (p.lse && lane == 0) *lse_of(p, b, qi, hk * p.g + hh) = log_of_sum(mm, ll);
  *reinterpret_cast<uint2*>(p.o + b * p.ob + qi * p.on + static_cast<int64_t>(hk * p.g + hh) * p.oh + lane * 4) =
      make_uint2(pack_bf16(a.x * r, a.y * r), pack_bf16(a.z * r, a.w * r));
}

int attn_kv4_cols(int columns) { return columns <= 8 ? 8 : 16; }

namespace {
template <int D, int G, int NT>
constexpr size_t ak_smem() {
  const size_t ring = static_cast<size_t>(AK_WARPS) * KvLayout<D, G>::RING;
  const size_t join = static_cast<size_t>(AK_WARPS) * 8 * NT * (D + 4 + 2) * 4;
  return ring > join ? ring : join;
}

template <int D, int G, int NT>
cudaError_t ak_run(const Kv4AttnParams& p, cudaStream_t s) {
  auto kern = p.solo ? attn_kv4_kernel<D, G, NT, true> : attn_kv4_kernel<D, G, NT, false>;
  constexpr size_t smem = ak_smem<D, G, NT>();
  cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), smem);
  if (e != cudaSuccess) return e;
  e = launch_following(kern, dim3(static_cast<unsigned>(p.ctas)), AK_THREADS, smem, s, p);
  if (e != cudaSuccess || p.block >= p.max_len || p.ctas == 1) return e;
  const int64_t items = static_cast<int64_t>(p.B) * p.Hk * p.n * p.g;
  // pieces of a sequence and head, about: CTAs per (sequence, head, chunk)
  if (p.ctas >= 4LL * p.B * p.Hk * p.col_chunks)
    return launch_following(attn_kv4_join_kernel<D, 8>, dim3(static_cast<unsigned>(items)), 256, 0, s, p, 8 * NT, p.ctas);
  return launch_following(attn_kv4_join_kernel<D, 1>, dim3(static_cast<unsigned>((items + 3) / 4)), 128, 0, s, p, 8 * NT, p.ctas);
}

template <int D, int G>
cudaError_t ak_cols(const Kv4AttnParams& p, cudaStream_t s) {
  return attn_kv4_cols(p.n * p.g) == 8 ? ak_run<D, G, 1>(p, s) : ak_run<D, G, 2>(p, s);
}
}  // namespace

int attn_kv4_resident(int head_dim, int group, int cols) { return ak_blocks(head_dim, group, cols / 8); }

cudaError_t launch_attn_kv4(const Kv4AttnParams& p, int D, int G, cudaStream_t s) {
  if (D == 64) return G == 32 ? ak_cols<64, 32>(p, s) : ak_cols<64, 64>(p, s);
  if (D == 96) return ak_cols<96, 32>(p, s);
  return G == 32 ? ak_cols<128, 32>(p, s) : G == 64 ? ak_cols<128, 64>(p, s) : ak_cols<128, 128>(p, s);
}

}  // namespace gc
