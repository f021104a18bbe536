// Attention of chunks of new tokens over the paged 4-bit cache: any number of query rows per sequence, packed one behind the other.
//
//   O = softmax(scale Q K^T) V, blockwise over 128 keys with a running reference, as in the prompt attention, K, V = lo + code * scale
//
// The products are tcgen05's with fp32 accumulators and fp16 operands: K, V and the probabilities are rounded once, to eleven bits.  (In bf16 the
// rounding of K alone puts the output off by 3-5e-3 of its norm, which is mostly cancellation, where the output's own rounding is 1.7e-3.)  Q, bf16,
// becomes fp16 after a warp's 32 rows are scaled by one power of two: exactly down to 2^-31 of their largest element, with an error of
// 2^-39 of it below; probabilities, at most 2^4 relative to the reference, are lifted by 2^11.
// K and V so small that fp16 has few bits left for them are widened in units of a power of two, one for each of the two and a CTA's part of an
// item, which the factor of the scores, and that of O at the end, make up for.  Where a part's first block is of ordinary size the unit is 1
// and nobody looks any further (22.7 -> 23.0 us for four short sequences, 176 -> 179 and 317 -> 320 for the two calls
// below); else the widening
// warps look through the parameters of all of its blocks first (values of 2^-20 throughout: 28, 206 and 363 us).  Units that change along a part,
// as larger values come, cost the ordinary case more than that: 415 us for the last, for what the softmax has to look at in every block.
//
// A row is a (token, query head) of those that share a key/value head, token by token, so that a block of keys, once widened, serves
// all of them.  A CTA holds 256 rows in two tiles of 128, and per block of 128 keys at width 128 there are
// two products of 512 clocks for each tile (2048 in all), as many clocks of exponentials (16 a clock), and 32768 elements to be
// widened: 3.4 instructions for two of them, 440 of the 2048 issue slots of a scheduler.
//   warps 0-3, 4-7   softmax of tile 0 / 1, one row per thread, 64 keys at a time: each half of a block's scores has its own place in
//                    tensor memory, barriers and products, its probabilities lie over it
//   warps 8-11       widen: codes and parameters out of staging, as fp16 into 128-byte-swizzled tiles of a ring.  The eight elements of a word
//                    come apart as (0,4), (1,5), (2,6), (3,7) and stay in that order: Q's elements are put in the same one, and
//                    the columns of O are put back in registers at the end.
//   warps 12, 13     MMA issuers of tile 0 / 1.  Only products into one accumulator, of one shape, are promised to keep their order: scores are
//                    multiplied only once the product that reads the probabilities they overwrite is complete.
//   warp 14          notes down which pieces of split items this CTA leaves
//   warp 15          bulk copies of codes and parameters, as they lie in the pages, a block and a half ahead (at width 64 four blocks); six
//                    blocks ahead they are called into the L2
// Where an item has at most 128 rows the two tiles are the same rows: they take the even and the odd blocks of keys, and
// are joined at the end, the one reading the other's O from tensor memory.
// The work is a row of units (three for a block of keys of an item, two where its tiles are twins, and six for its beginning; an item is
// 256 rows of a sequence, times heads), of which every CTA takes an equal stretch; the pieces of an item that stretches cut are joined in their order by a second kernel.
//   * A value that is not finite must not reach rows that do not see it (0 times NaN): such groups are widened as zeros and
//     noted in a bit mask per block; a row that does see one gets NaN in that group's columns.
//
// Measured, calls in a row: the last 1024 tokens of a sequence of 33001, 16 / 4 heads of 128 (0.27 TFLOP): 317 to 334 us from one GPU to another,
// 860 to 815 TFLOP/s; 32 sequences of up to 4096, chunks of up to 192 tokens, three in four of one, 32 / 8 heads of 128: 179 us.  Tensor pipe 41 %, XU 41 %, ALU
// 42 %, half an instruction a clock and scheduler of one: no unit is at its limit; the time goes into the way round of a half block, products,
// exponentials, probabilities, products, with two halves of two tiles under way (without any arithmetic the handshakes alone took 127 of
// 318).  At widths 96 and 128 reading and scaling Q spills 360 to 420 bytes a thread, at an item's beginning.  Tried for the first of these calls, then 318: 128 scores
// in registers, unrolled, with registers moved between warps 368 (its code no longer fits the instruction cache); two groups of
// softmax warps for each tile 359; eight widening warps 347; tiles taking turns 370; staging by loads through the cores 342.
#include <cuda_fp16.h>

#include <type_traits>

#include "attn_tc.cuh"
#include "ptx.cuh"
#include "serving.cuh"

namespace gc {

namespace {
constexpr int CK_THREADS = 512, CK_ROWS = 256;
constexpr int CK_MAX_LIST = 160;             // items per head that are listed in shared memory
constexpr int CK_START = 6, CK_BLOCK = 3, CK_TWIN_BLOCK = 2;      // what beginning an item and a block of its keys cost, in units of about 1700 clocks
// A CTA takes at least this many units.  The joining kernel reads a piece of every CTA between an item's first and last, so that a
// stretch has to have some block's first unit in it, wherever it begins inside an item.
constexpr int CK_LEAST = 4;
static_assert(CK_LEAST >= CK_BLOCK && CK_LEAST >= CK_TWIN_BLOCK, "a stretch could lie inside one block, and its piece would not be written");
constexpr int CK_FETCH = 6;                  // blocks of keys that are called into the L2 ahead of their copies
constexpr int CK_FLAGS = 8;                  // blocks whose notes of values that are not finite are kept
constexpr float CK_RAISE = 4.0f;             // binades a score may exceed the reference by
constexpr float CK_LIFT = 11.0f;             // binades the probabilities are lifted by: at most 2^15, and whole down to 2^-25 of the reference
constexpr float CK_LARGEST = 65504.0f;       // the largest fp16
// Keys and values whose largest lies below 2^CK_SMALL are widened in units of 2^-CK_MOST_UNIT at least, in which it lies from 2^CK_TOP to twice
// that.  (A value is off by half a step, or by 2^-25 where that is more, and as much for lo and 15 times as much for its scale, which
// are rounded first: by 17 2^-25 in all, or 17 2^-38 of the largest.)
constexpr int CK_SMALL = -8, CK_TOP = 13, CK_MOST_UNIT = 100;
template <int D, int G>
struct ChunkLayout {
  static constexpr int NSUB = (D + 63) / 64;     // 64-element sub-tiles of 128-byte rows
  static constexpr int SUB = 128 * 128;
  static constexpr int TILE = NSUB * SUB;        // 128 rows of Q, K or V
  static constexpr int STAGES = D == 64 ? 8 : 4;
  // codes and parameters of 128 key rows, K's or V's, as they lie in memory, and how many of these there are
  static constexpr int NG = D / G, PITCH = D / 2, CODES = 128 * PITCH, STAGED = CODES + 128 * NG * 4, AHEAD = D == 64 ? 8 : 3;
  static constexpr int BARS = 2 * STAGES + 2 * AHEAD + 17;
  // Q, ring, staged codes, list, notes [CK_FLAGS][4 groups][4 words], one word a block that sums them up, one a part with its units, the widening
  // warps' sizes [2][4], sums of the second tile [3][128]
  static constexpr int LIST = CK_MAX_LIST * 8, NOTES = CK_FLAGS * 16 * 4, ANY = CK_FLAGS * 4, UNITS = CK_FLAGS * 4 + 2 * 4 * 4, SUMS = 3 * 128 * 4;
  static constexpr size_t SMEM = 1024 + static_cast<size_t>(2 + STAGES) * TILE + AHEAD * STAGED + LIST + NOTES + ANY + UNITS + SUMS + BARS * 8 + 64 * 4;
};

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ __half2 half2_of(uint32_t w) { return *reinterpret_cast<const __half2*>(&w); }
// The parameters (lo, scale) of a group in fp16, lo and scale twice each; false where a value of the group is not finite in fp16
// (a straight line in the code: its ends are what to look at).
struct Params16 {
  uint32_t lo2, scale2;
};
__device__ __forceinline__ bool fits_half(uint32_t par, uint32_t* status) {
  const float lo = __uint_as_float(par << 16), scale = __uint_as_float(par & 0xffff0000u);
  if (fabsf(lo) <= CK_LARGEST && fabsf(fmaf(15.f, scale, lo)) <= CK_LARGEST && fabsf(scale) <= CK_LARGEST) return true;
  if (fabsf(lo) < INFINITY && fabsf(scale) < INFINITY) report(status, DEV_LARGE_HALF);
  return false;
}
// (by: what they are multiplied by, a power of two)
__device__ __forceinline__ Params16 params16(uint32_t par, float by) {
  const float l = __uint_as_float(par << 16) * by, c = __uint_as_float(par & 0xffff0000u) * by;
  const uint32_t lo = pack_half(l, l), scale = pack_half(c, c);
  return Params16{lo, scale};
}

// Bulk copy global -> shared of a multiple of 16 bytes, completion counted in bytes on an mbarrier of this CTA.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred P;\n\tmbarrier.test_wait.parity.shared::cta.b64 P, [%1], %2;\n\tselp.b32 %0, 1, 0, P;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ void bulk_prefetch(const void* src, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}

// The largest finite element in size of a warp's rows, one offset a lane (-1: none).  (A call: inline it takes registers of every block, 183 us for 176.)
template <int D>
__device__ __noinline__ float largest_finite(const __nv_bfloat16* q, int64_t offset, int lane) {
  float top = 0.f;
#pragma unroll 1
  for (int r = 0; r < 32; ++r) {
    const int64_t at = __shfl_sync(0xffffffffu, offset, r);
#pragma unroll 1
    for (int i = lane; i < D && at >= 0; i += 32) {
      const float v = fabsf(__bfloat162float(q[at + i]));
      if (v < INFINITY) top = fmaxf(top, v);
    }
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  return top;
}

// One sequence: its query rows, and the tokens it has cached.
struct ChunkSeq {
  int q0, nq, len;
};
__device__ __forceinline__ ChunkSeq seq_of(const ChunkParams& p, int b) {
  ChunkSeq s;
  const int tq = static_cast<int>(p.q_tokens);
  s.q0 = min(max(p.cu_q[b], 0), tq);
  s.nq = max(min(p.cu_q[b + 1], tq) - s.q0, 0);
  s.len = min(max(p.lengths[b], 0), p.max_len);
  return s;
}
__device__ __forceinline__ int items_of(const ChunkParams& p, const ChunkSeq& s) { return (s.nq * p.g + CK_ROWS - 1) / CK_ROWS; }
// Blocks of keys that item number i of a sequence needs; at least one, so that rows which see nothing are written as well.
__device__ __forceinline__ int blocks_of(const ChunkParams& p, const ChunkSeq& s, int i) {
  const int last = (min((i + 1) * CK_ROWS, s.nq * p.g) - 1) / p.g;       // token of the last row
  return (max(min(s.len - s.nq + last + 1, s.len), 1) + 127) >> 7;
}

__device__ __forceinline__ int block_cost(int rows) { return rows <= 128 ? CK_TWIN_BLOCK : CK_BLOCK; }

// An item of the list: the units before it, its sequence and its number there.
struct Entry {
  int before, b, i;
};
// The list in shared memory packs sequence and number, both below CK_MAX_LIST, into a word.
struct ListShared {
  uint2* at;
  __device__ __forceinline__ Entry get(int e) const {
    const uint2 x = at[e];
    return Entry{static_cast<int>(x.x), static_cast<int>(x.y >> 16), static_cast<int>(x.y & 0xffffu)};
  }
  __device__ __forceinline__ void put(int e, int cost, int b, int i) const { at[e] = make_uint2(static_cast<uint32_t>(cost), static_cast<uint32_t>(b) << 16 | static_cast<uint32_t>(i)); }
  __device__ __forceinline__ int cost(int e) const { return static_cast<int>(at[e].x); }
  __device__ __forceinline__ void before(int e, int units) const { at[e].x = static_cast<uint32_t>(units); }
};
struct ListGlobal {
  int4* at;
  __device__ __forceinline__ Entry get(int e) const {
    const int4 x = at[e];
    return Entry{x.x, x.y, x.z};
  }
  __device__ __forceinline__ void put(int e, int cost, int b, int i) const { at[e] = make_int4(cost, b, i, 0); }
  __device__ __forceinline__ int cost(int e) const { return at[e].x; }
  __device__ __forceinline__ void before(int e, int units) const { at[e].x = units; }
};

// Sum of v over the threads before this one, and over all; called by all CK_THREADS threads.
__device__ __forceinline__ int block_scan(int v, int* s_sums, int* all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  __syncthreads();
  if (lane == 31) s_sums[warp] = incl;
  __syncthreads();
  int before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < CK_THREADS / 32; ++w) {
    const int x = s_sums[w];
    if (w < warp) before += x;
    total += x;
  }
  *all = total;
  return before + incl - v;
}
// Makes the list (never more than `most` items: offsets that overlap, an error, could ask for more); returns items and units.
// s_seq: scratch, one entry a thread.
template <typename List>
__device__ int2 make_list(const ChunkParams& p, const List& list, int most, int* s_sums, int4* s_seq) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int items = 0;
#pragma unroll 1
  for (int s0 = 0; s0 < p.B; s0 += CK_THREADS) {
    const int b = s0 + tid, here = min(p.B - s0, CK_THREADS);
    int count = 0;
    ChunkSeq s = {};
    if (tid < here) {
      s = seq_of(p, b);
      count = items_of(p, s);
      if (blockIdx.x == 0) {
        if (p.cu_q[b] != s.q0 || p.cu_q[b + 1] != s.q0 + s.nq) report(p.status, DEV_BAD_OFFSETS);
        if (p.lengths[b] != s.len) report(p.status, DEV_BAD_LENGTH);
      }
    }
    int all;
    const int before = block_scan(count, s_sums, &all);
    s_seq[tid] = make_int4(items + before, s.nq, s.len, count);
    __syncthreads();
#pragma unroll 1
    for (int w = warp; w < here; w += CK_THREADS / 32) {
      const int4 x = s_seq[w];
#pragma unroll 1
      for (int i = lane; i < x.w && x.x + i < most; i += 32) list.put(x.x + i, blocks_of(p, ChunkSeq{0, x.y, x.z}, i) * block_cost(min(x.y * p.g - i * CK_ROWS, CK_ROWS)) + CK_START, s0 + w, i);
    }
    items = min(items + all, most);
    __syncthreads();
  }
  int units = 0;
#pragma unroll 1
  for (int e0 = 0; e0 < items; e0 += CK_THREADS) {
    const int e = e0 + tid, cost = e < items ? list.cost(e) : 0;
    int all;
    const int before = block_scan(cost, s_sums, &all);
    if (e < items) list.before(e, units + before);
    units += all;
  }
  __syncthreads();
  return make_int2(items, units);
}

// (A division of 64-bit numbers costs hundreds of clocks, and most are small.)
__device__ __forceinline__ int64_t quotient(int64_t a, int b) {
  return (a >> 32) == 0 ? static_cast<int64_t>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b)) : a / b;
}
// Where CTA number c's stretch begins.
struct Cuts {
  int64_t each;
  int rest;
  __device__ __forceinline__ Cuts(int64_t total, int ctas) : each(quotient(total, ctas)), rest(static_cast<int>(total - each * ctas)) {}
  __device__ __forceinline__ int64_t at(int c) const { return each * c + min(c, rest); }
};

// Part of an item: blocks [j0, j1) of its n; a CTA's stretch is a sequence of them.
struct Seg {
  int b, h, row0, rows, q0, len, ahead;      // row0: first row in the sequence; ahead: tokens before the new ones
  int j0, j1, n;
  __device__ __forceinline__ bool twin() const { return rows <= 128; }
  __device__ __forceinline__ bool whole() const { return j0 == 0 && j1 == n; }
};
template <typename List>
struct Walk {
  const ChunkParams& p;
  const List& list;
  int items, units;
  int64_t left;
  int e, h, j;
  __device__ __forceinline__ Walk(const ChunkParams& p_, const List& l, int items_, int units_, int64_t from, int64_t to)
      : p(p_), list(l), items(items_), units(units_), left(to - from) {
    if (left <= 0) return;
    h = static_cast<int>(quotient(from, units));
    const int at = static_cast<int>(from - static_cast<int64_t>(h) * units), lane = threadIdx.x & 31;
    // the last item that does not begin behind `at`, 32 places at a time (whole warps make a walk together)
    int lo = 0, n = items;
#pragma unroll 1
    while (n > 1) {
      const int step = (n + 31) >> 5, i = lane * step;
      const uint32_t hit = __ballot_sync(0xffffffffu, i < n && list.get(lo + min(i, n - 1)).before <= at);
      const int last = __popc(hit) - 1;
      lo += last * step;
      n = min(step, n - last * step);
    }
    e = lo;
    j = at - list.get(e).before;
  }
  __device__ __forceinline__ bool next(Seg& s) {
    while (left > 0) {
      const Entry x = list.get(e);
      const ChunkSeq q = seq_of(p, x.b);
      s.h = h;
      s.row0 = x.i * CK_ROWS;
      s.rows = min(q.nq * p.g - s.row0, CK_ROWS);
      s.q0 = q.q0;
      s.len = q.len;
      s.ahead = q.len - q.nq;
      s.b = x.b;
      s.n = blocks_of(p, q, x.i);
      const int cost = block_cost(s.rows), take = static_cast<int>(min(static_cast<int64_t>(s.n * cost + CK_START - j), left));
      // (a block belongs to the stretch that has its first unit)
      s.j0 = (max(j - CK_START, 0) + cost - 1) / cost;
      s.j1 = (max(j + take - CK_START, 0) + cost - 1) / cost;
      left -= take;
      j = 0;
      if (++e == items) {
        e = 0;
        ++h;
      }
      if (s.j1 > s.j0) return true;                              // (else the stretch ends before the item's first block)
    }
    return false;
  }
};

// What a CTA leaves to the joining kernel: a piece that begins an item without reaching its end (slot 1; rows > 0), and one that
// begins inside an item (slot 0), which may reach its end.
struct Note {
  int rows, q0, row0, h;
  int ends, pad[3];
};

// 2^n for n from -126 to 127.
__device__ __forceinline__ float exp2_of(int n) { return __uint_as_float(static_cast<uint32_t>(127 + n) << 23); }
// What the values of a group do not exceed in size, as bits; zero where they are not finite.
__device__ __forceinline__ uint32_t size_of(uint32_t par) {
  const float u = fmaf(16.f, fabsf(__uint_as_float(par & 0xffff0000u)), fabsf(__uint_as_float(par << 16)));
  return u < INFINITY ? __float_as_uint(u) : 0u;
}
// u for units of 2^-u.
__device__ __forceinline__ bool is_small(uint32_t size) { return size < static_cast<uint32_t>(127 + CK_SMALL) << 23; }
__device__ __forceinline__ uint32_t unit_of(uint32_t size) {
  return size == 0 || !is_small(size) ? 0u : static_cast<uint32_t>(min(CK_TOP + 127 - static_cast<int>(size >> 23), CK_MOST_UNIT));
}
// The unit of the keys, or values, of a part of an item, whose first block's parameters are staged at `staged`.  A widening warp that finds all that it
// has of that block small calls this (out of line: their loop is at its best when it is short).  Where the whole block is, and others follow, all
// four do, and each looks through a quarter of the rows; *looks: how often they have.  `sizes` [2][4], and a barrier of four arrivals.
constexpr uint32_t NO_UNIT = 0xffffffffu;    // a wait ran out
template <int D, int G>
__device__ __noinline__ uint32_t unit_of_part(const ChunkParams& p, const uint32_t* params, uint32_t staged, uint32_t* sizes, uint32_t bar, uint32_t* looks, int b, int h,
                                              int j0, int j1, int len, int warp, int lane) {
  constexpr int NG = D / G, FLY = 8;
  uint32_t size = 0;
  for (int i = lane; i < 128 * NG; i += 32)
    if (i / NG < len - j0 * 128) size = max(size, size_of(lds32(staged + i * 4)));
  size = __reduce_max_sync(0xffffffffu, size);
  if (!is_small(size)) return 0;
  if (j1 - j0 == 1) return unit_of(size);
  const int* table = p.table + b * p.table_stride;
  const int end = min(j1 * 128, len);
#pragma unroll 1
  for (int t0 = (j0 + 1) * 128 + warp * 32 + lane; t0 < end; t0 += 128 * FLY) {
    int64_t at[FLY];
#pragma unroll
    for (int k = 0; k < FLY; ++k) {
      const int t = t0 + k * 128, page = t < end ? table[t >> p.page_shift] : -1;
      // (a page that is none is reported where it is copied)
      at[k] = page < 0 || page >= p.num_pages ? -1 : ((static_cast<int64_t>(page) * p.Hk + h) << p.page_shift) + (t & ((1 << p.page_shift) - 1));
    }
    uint32_t x[FLY][NG];
#pragma unroll
    for (int k = 0; k < FLY; ++k) {
#pragma unroll
      for (int g = 0; g < NG; ++g) x[k][g] = at[k] < 0 ? 0 : params[at[k] * NG + g];
    }
#pragma unroll
    for (int k = 0; k < FLY; ++k) {
#pragma unroll
      for (int g = 0; g < NG; ++g) size = max(size, size_of(x[k][g]));
    }
  }
  size = __reduce_max_sync(0xffffffffu, size);
  // (The next look's go into the other four places; those of the one after only come once all have arrived for that.)
  const uint32_t look = (*looks)++;
  uint32_t* mine = sizes + (look & 1) * 4;
  if (lane == 0) {
    mine[warp] = size;
    mbar_arrive(bar);
  }
  if (!__all_sync(0xffffffffu, mma_wait(bar, look & 1))) return NO_UNIT;
  return unit_of(max(max(mine[0], mine[1]), max(mine[2], mine[3])));
}
}  // namespace

// Workspace: pieces [ctas][2][D / 4][256] of four columns, their (reference, sum) [ctas][2][256], notes [ctas], and the list
// (items and units, then the items) where it does not fit shared memory.
template <int D>
struct ChunkSpace {
  float4* o;
  float2* ml;
  Note* note;
  int4* list;
  __host__ __device__ ChunkSpace(void* ws, int ctas) {
    o = static_cast<float4*>(ws);
    ml = reinterpret_cast<float2*>(o + static_cast<int64_t>(ctas) * 2 * (D / 4) * CK_ROWS);
    note = reinterpret_cast<Note*>(ml + static_cast<int64_t>(ctas) * 2 * CK_ROWS);
    list = reinterpret_cast<int4*>(note + ctas);
  }
};

template <int D>
__global__ void __launch_bounds__(CK_THREADS, 1) attn_chunk_list_kernel(const __grid_constant__ ChunkParams p, const int ctas) {
  __shared__ int s_sums[CK_THREADS / 32];
  __shared__ int4 s_seq[CK_THREADS];
  wait_for_predecessor();
  int4* list = ChunkSpace<D>(p.ws, ctas).list;
  const int2 got = make_list(p, ListGlobal{list + 1}, p.most_items, s_sums, s_seq);
  if (threadIdx.x == 0) list[0] = make_int4(got.x, got.y, 0, 0);
}

template <int D, int G, typename List>
__global__ void __launch_bounds__(CK_THREADS, 1) attn_chunk_kernel(const __grid_constant__ ChunkParams p) {
  using L = ChunkLayout<D, G>;
  static_assert(L::SMEM <= 232448, "more than an SM's shared memory");
  constexpr int NG = D / G;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = smem;                                           // [2] tiles
  uint8_t* sKV = sQ + 2 * L::TILE;                              // [STAGES] tiles
  uint8_t* s_staging = sKV + L::STAGES * L::TILE;
  uint2* s_list = reinterpret_cast<uint2*>(s_staging + L::AHEAD * L::STAGED);
  uint32_t* s_notes = reinterpret_cast<uint32_t*>(s_list + CK_MAX_LIST);        // [CK_FLAGS][4][4]
  uint32_t* s_any = s_notes + CK_FLAGS * 16;                    // [CK_FLAGS], a byte per widening warp
  uint32_t* s_units = s_any + CK_FLAGS;                         // [CK_FLAGS] parts of items: bytes of K and V
  uint32_t* s_sizes = s_units + CK_FLAGS;                       // [2][4]
  float* s_second = reinterpret_cast<float*>(s_sizes + 8);      // reference, sum and groups that are not finite of tile 1
  uint64_t* bars = reinterpret_cast<uint64_t*>(s_second + 3 * 128);
  const uint32_t b0 = smem_u32(bars);
  const uint32_t bar_q_full = b0, bar_q_empty = b0 + 8, bar_s_full = b0 + 16, bar_p_full = b0 + 48, bar_o_full = b0 + 80;
  const uint32_t bar_second = b0 + 112, bar_joined = b0 + 120, bar_kv_full = b0 + 128, bar_kv_empty = bar_kv_full + 8 * L::STAGES;
  const uint32_t bar_code_full = bar_kv_empty + 8 * L::STAGES, bar_code_empty = bar_code_full + 8 * L::AHEAD;
  const uint32_t bar_sizes = bar_code_empty + 8 * L::AHEAD;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + L::BARS);
  int* s_sums = reinterpret_cast<int*>(tmem_slot + 4);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    mbar_init(bar_q_full, 8);                                   // the softmax warps
    mbar_init(bar_q_empty, 2);                                  // both tiles' issuers
    mbar_init(bar_second, 4);
    mbar_init(bar_joined, 4);
    mbar_init(bar_sizes, 4);                                    // the widening warps
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar_s_full + 8 * i, 1);
      mbar_init(bar_o_full + 8 * i, 1);
      mbar_init(bar_p_full + 8 * i, 4);
    }
    for (int i = 0; i < L::STAGES; ++i) {
      mbar_init(bar_kv_full + 8 * i, 4);
      mbar_init(bar_kv_empty + 8 * i, 2);
    }
    for (int i = 0; i < L::AHEAD; ++i) {
      mbar_init(bar_code_full + 8 * i, 1);
      mbar_init(bar_code_empty + 8 * i, 4);
    }
    fence_mbar_init();
  }
  if (warp == 12) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int ctas = static_cast<int>(gridDim.x);
  const ChunkSpace<D> space(p.ws, ctas);
  List list;
  int2 size;
  if constexpr (std::is_same<List, ListShared>::value) {
    list.at = s_list;
    size = make_list(p, list, CK_MAX_LIST, s_sums, reinterpret_cast<int4*>(sQ));
  } else {
    list.at = space.list + 1;
    size = make_int2(space.list[0].x, space.list[0].y);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // Not before this block has its tensor memory: a block of the next kernel that took the columns first would wait for this
  // kernel's end, and this one for the columns.
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t tmem_base = *tmem_slot;
  // Stretches of at least CK_LEAST units: fewer CTAs work where there is little to do.
  const int64_t total = static_cast<int64_t>(size.y) * p.Hk;
  const int64_t fill = quotient(total, CK_LEAST);
  const int working = fill < ctas ? max(static_cast<int>(fill), 1) : ctas, me = static_cast<int>(blockIdx.x);
  const Cuts cuts(total, working);
  Walk<List> walk(p, list, size.x, size.y, me < working ? cuts.at(me) : 0, me < working ? cuts.at(me + 1) : 0);

  bool failed = false;
  if (warp < 8) {
    // ------------------------------------------------------------------ softmax and output
    const int t = warp >> 2, row = tid & 127;
    const uint32_t t_lane = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t s_addr = t_lane + t * 128, o_addr = t_lane + 256 + t * 128;
    uint32_t sn = 0, jn = 0, qn = 0, block = 0;                 // block: number of the segment's first among all of this CTA's
    Seg s;
    while (!failed && walk.next(s)) {
      const bool twin = s.twin();
      const int my_row = s.row0 + (twin ? row : t * 128 + row);
      const bool mine = my_row < s.row0 + s.rows;
      const int token = mine ? my_row / p.g : 0;
      const int lim = mine ? max(min(s.ahead + token + 1, s.len), 0) : 0;
      const int j_first = twin ? s.j0 + t : s.j0, j_step = twin ? 2 : 1;
      float m = -INFINITY, l = 0.f, factor = 0.f;
      uint32_t poison = 0;                                      // groups of columns in which this row saw a value that is not finite
      int seen_blocks = 0;
      // ---- Q: fp16 after scaling by a power of two, so that the largest element of this warp's 32 rows lies in [2^14, 2^15).  A row is read
      // by 16 (at width 64: 8) neighbouring lanes, all rows at once.  (Scaled row by row: 5 us a segment where this takes 2.)
      constexpr int LPR = D == 64 ? 8 : 16, RPI = 32 / LPR, N = 32 / RPI;        // lanes to a row, rows to a load, loads
      const int lc = lane % LPR, lr = lane / LPR;
      const int64_t my_head = mine ? static_cast<int64_t>(s.h * p.g + my_row - token * p.g) : -1;
      {
        const int64_t my_offset = mine ? static_cast<int64_t>(s.q0 + token) * p.q_tok + my_head * p.q_head : -1;
        uint4 x[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int64_t at = __shfl_sync(0xffffffffu, my_offset, i * RPI + lr);
          x[i] = make_uint4(0, 0, 0, 0);
          if (at >= 0 && lc < D / 8) x[i] = reinterpret_cast<const uint4*>(p.q + at)[lc];
        }
        float tops[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) tops[e] = max3(tops[e], fabsf(__uint_as_float(w[e] << 16)), fabsf(__uint_as_float(w[e] & 0xffff0000u)));
        }
        float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
#pragma unroll
        for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        if (top == INFINITY) {                                  // it stays one; the other rows' scale must not go by it
          top = largest_finite<D>(p.q, my_offset, lane);
        }
        // (zeros: as they are; rows below 2^-86 need not keep their eight bits, for their scores are nothing)
        const int ex = static_cast<int>(__float_as_uint(top) >> 23), e = top == 0.f ? 0 : max(ex - 141, -100);
        const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
        factor = p.c * __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
        if (!__all_sync(0xffffffffu, mma_wait(bar_q_empty, (qn & 1) ^ 1))) { failed = true; break; }
        ++qn;
        if (!(twin && t) && lc < D / 8) {
          uint8_t* tile = sQ + t * L::TILE + (warp & 3) * 32 * 128 + (lc >> 3) * L::SUB;
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
            float v[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              v[2 * k] = __uint_as_float(w[k] << 16) * down;
              v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u) * down;
            }
            const int r = i * RPI + lr;
            *reinterpret_cast<uint4*>(tile + r * 128 + (((lc ^ r) & 7) << 4)) = make_uint4(pack_half(v[0], v[4]), pack_half(v[1], v[5]), pack_half(v[2], v[6]), pack_half(v[3], v[7]));
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_q_full);
      }
      // The unit of this part's keys is known once they have been widened, as the first scores show (tile 1 may have none).
      if (j_first < s.j1 && !__all_sync(0xffffffffu, mma_wait(bar_s_full + 16 * t, sn & 1))) { failed = true; break; }
      // c times the power of two the scores are short of
      const float c = factor * exp2_of(-static_cast<int>(reinterpret_cast<const volatile uint8_t*>(s_units + (qn - 1) % CK_FLAGS)[0]));
      // What was noted of block j's values, once a product that waited for them is known to be issued; they are overwritten eight blocks
      // on, when all rows have handed over probabilities made after this look.
      auto look = [&](int j) {
        const uint32_t slot = (block + j - s.j0) % CK_FLAGS;
        const uint32_t any = s_any[slot];
        if (any == 0) return;
#pragma unroll 1
        for (int x = 0; x < 4 * NG; ++x) {
          const int g = x >> 2, w = x & 3, k = lim - j * 128 - 32 * w;
          const uint32_t sees = k >= 32 ? 0xffffffffu : k <= 0 ? 0u : (1u << k) - 1u;
          // (only the warps that found something have written their words)
          if ((any >> (8 * w) & 0xffu) && (s_notes[slot * 16 + g * 4 + w] & sees)) poison |= 1u << g;
        }
      };
#pragma unroll 1
      for (int x = 0; j_first + (x >> 1) * j_step < s.j1; ++x) {
        const int j = j_first + (x >> 1) * j_step, h = x & 1;
        if (!__all_sync(0xffffffffu, mma_wait(bar_s_full + 8 * (2 * t + h), sn & 1))) { failed = true; break; }
        // the product before these scores: complete with them, but no phase of a barrier may be left out
        if (x >= 2 && !__all_sync(0xffffffffu, mma_wait(bar_o_full + 8 * (2 * t + h), (sn - 1) & 1))) { failed = true; break; }
        tc_fence_after();
        uint32_t v[64];
        tmem_ld64(s_addr + h * 64, v);
        if (h == 0 && seen_blocks) look(j - j_step);
        const int left = lim - j * 128 - h * 64;
        if (__any_sync(0xffffffffu, left < 64)) {
#pragma unroll
          for (int i = 0; i < 64; ++i)
            if (i >= left) v[i] = 0xff800000u;                   // minus infinity, whatever the score was
        }
        float top[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) top[i] = max3(__uint_as_float(v[16 * i]), __uint_as_float(v[16 * i + 1]), -INFINITY);
#pragma unroll
        for (int i = 2; i < 16; i += 2) {
#pragma unroll
          for (int k = 0; k < 4; ++k) top[k] = max3(top[k], __uint_as_float(v[16 * k + i]), __uint_as_float(v[16 * k + i + 1]));
        }
        const float mx = max3(max3(top[0], top[1], top[2]), top[3], top[3]);
        if (__any_sync(0xffffffffu, (mx - m) * c > CK_RAISE)) {
          const float mn = fmaxf(m, mx);
          if (score_too_large(mn * c)) report(p.status, DEV_LARGE_SCORE);
          const float f = mn == m ? 1.f : ap_ex2((m - mn) * c);  // 0 from the initial minus infinity
          m = mn;
          l *= f;
          if (x > 0) {
            // the product of the half block before: O is at rest
            if (!__all_sync(0xffffffffu, mma_wait(bar_o_full + 8 * (2 * t + (h ^ 1)), (sn - (h ^ 1)) & 1))) { failed = true; break; }
            tc_fence_after();
#pragma unroll 1
            for (int k = 0; k < D / 16; ++k) {
              uint32_t w[16];
              tmem_ld16(o_addr + k * 16, w);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(__uint_as_float(w[i]) * f);
              tmem_st16(o_addr + k * 16, w);
            }
          }
        }
        const float off = m == -INFINITY ? 0.f : fmaf(-m, c, CK_LIFT);
        const uint64_t c2 = pair2(c, c), off2 = pair2(off, off);
        uint64_t ls[2] = {0, 0};
        uint32_t w[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          float e0, e1;
          unpair2(fma2(pair2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), c2, off2), &e0, &e1);
          e0 = ap_ex2(e0);
          e1 = ap_ex2(e1);
          ls[i & 1] = add2(ls[i & 1], pair2(e0, e1));
          w[i] = pack_half(e0, e1);
        }
        tmem_st32(s_addr + h * 64, w);                           // over the scores
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_p_full + 8 * (2 * t + h));
        float l0, l1;
        unpair2(add2(ls[0], ls[1]), &l0, &l1);
        l += l0 + l1;
        sn += h;
        seen_blocks += h;
      }
      if (failed) break;
      if (seen_blocks) {
        if (!__all_sync(0xffffffffu, mma_wait(bar_o_full + 16 * t, (sn - 1) & 1) && mma_wait(bar_o_full + 16 * t + 8, (sn - 1) & 1))) { failed = true; break; }
        tc_fence_after();
        look(j_first + (seen_blocks - 1) * j_step);
      }
      block += s.j1 - s.j0;
      float f0 = 1.f, f1 = 0.f;
      bool second = false;                                      // tile 1 has a part of these rows
      if (twin && t == 1) {
        // O of this tile is complete: tile 0 may take it
        s_second[row] = m;
        s_second[128 + row] = l;
        s_second[256 + row] = __uint_as_float(poison);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_second);
        if (!__all_sync(0xffffffffu, mma_wait(bar_joined, jn & 1))) { failed = true; break; }
        ++jn;
        tc_fence_after();
        continue;
      }
      if (twin) {
        if (!__all_sync(0xffffffffu, mma_wait(bar_second, jn & 1))) { failed = true; break; }
        ++jn;
        tc_fence_after();
        second = s.j1 - s.j0 > 1;
        const float m1 = s_second[row], l1 = s_second[128 + row];
        poison |= __float_as_uint(s_second[256 + row]);
        const float mm = fmaxf(m, m1), ref = mm == -INFINITY ? 0.f : mm;
        f0 = ap_ex2((m - ref) * c);                             // 0 from minus infinity; NaN sums pass
        f1 = ap_ex2((m1 - ref) * c);
        l = second ? fmaf(f0, l, f1 * l1) : f0 * l;
        m = mm;
      }
      const float fall = exp2_of(-static_cast<int>(reinterpret_cast<const volatile uint8_t*>(s_units + (qn - 1) % CK_FLAGS)[1]));
      const bool whole = s.whole();
      const float rl = l == 0.f ? 0.f : whole ? 1.0f / l : 1.f;
      const float a0 = f0 * rl * fall, a1 = f1 * rl * fall;
      const int64_t piece = 2 * static_cast<int64_t>(me) + (s.j0 == 0);
      const int my_slot = my_row - s.row0;
      float4* po = space.o + piece * (D / 4) * CK_ROWS + my_slot;
      // Rows go out through this warp's own rows of Q, which no product reads any more, in Q's layout.
      uint8_t* out = sQ + t * L::TILE + (warp & 3) * 32 * 128;
      if (!whole && mine) space.ml[piece * CK_ROWS + my_slot] = make_float2(m == -INFINITY ? -INFINITY : m * c, l);
#pragma unroll 1
      for (int k = 0; k < D / 32; ++k) {
        uint32_t w[32];
        tmem_ld32(o_addr + k * 32, w);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(__uint_as_float(w[i]) * a0);
        if (second) {
          uint32_t x[32];
          tmem_ld32(o_addr + 128 + k * 32, x);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(fmaf(__uint_as_float(x[i]), a1, __uint_as_float(w[i])));
        }
        if (poison >> (k * 32 / G) & 1u) {
#pragma unroll
          for (int i = 0; i < 32; ++i) w[i] = 0x7fffffffu;
        }
        {
          // back into order: columns 8 i + (0, 4, 1, 5, 2, 6, 3, 7)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float e[8] = {__uint_as_float(w[8 * i]), __uint_as_float(w[8 * i + 2]), __uint_as_float(w[8 * i + 4]), __uint_as_float(w[8 * i + 6]),
                                __uint_as_float(w[8 * i + 1]), __uint_as_float(w[8 * i + 3]), __uint_as_float(w[8 * i + 5]), __uint_as_float(w[8 * i + 7])};
            if (whole) {
              *reinterpret_cast<uint4*>(out + (k >> 1) * L::SUB + lane * 128 + ((((k & 1) * 4 + i) ^ (lane & 7)) << 4)) = make_uint4(ap_pack(e[0], e[1]), ap_pack(e[2], e[3]), ap_pack(e[4], e[5]), ap_pack(e[6], e[7]));
            } else if (mine) {
              po[(k * 8 + 2 * i) * CK_ROWS] = make_float4(e[0], e[1], e[2], e[3]);
              po[(k * 8 + 2 * i + 1) * CK_ROWS] = make_float4(e[4], e[5], e[6], e[7]);
            }
          }
        }
      }
      if (whole) {                                              // as Q was read
        const int64_t my_offset = mine ? static_cast<int64_t>(s.q0 + token) * p.o_tok + my_head * p.o_head : -1;
        __syncwarp();
#pragma unroll 2
        for (int i = 0; i < N; ++i) {
          const int r = i * RPI + lr;
          const int64_t at = __shfl_sync(0xffffffffu, my_offset, r);
          if (at >= 0 && lc < D / 8)
            reinterpret_cast<uint4*>(p.o + at)[lc] = *reinterpret_cast<const uint4*>(out + (lc >> 3) * L::SUB + r * 128 + (((lc ^ r) & 7) << 4));
        }
        __syncwarp();
      }
      tc_fence_before();
      if (twin) {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_joined);
      }
    }
    if (failed && lane == 0) report(p.status, DEV_TIMEOUT_EPILOGUE);
  } else if (warp < 12) {
    // ------------------------------------------------------------------ widening
    // A lane takes 16 bytes of codes (32 elements) of a row at a time, CH times.  At width 128 and 64 eight lanes take two neighbouring chunks
    // of four rows, so that the four stores of 16 bytes that become of each touch all banks; at 96 a lane takes a row, and the rows' pitch spreads
    // them.  Round k: 16 rows on, or two chunks on.
    constexpr int CH = D / 32;                                  // 16-byte chunks of codes in a row
    const int row0 = (warp & 3) * 32 + (D == 96 ? lane : ((lane >> 3) & 3) * 4 + ((lane >> 1) & 3)), chunk0 = D == 96 ? 0 : lane & 1;
    auto row_of = [&](int k) { return row0 + (D == 96 ? 0 : (k & 1) * 16); };
    auto chunk_of = [&](int k) { return chunk0 + (D == 96 ? k : (k >> 1) * 2); };
    const uint32_t code0 = smem_u32(s_staging) + row0 * L::PITCH + chunk0 * 16, par0 = smem_u32(s_staging) + L::CODES + row0 * NG * 4;
    uint32_t to[4];                                             // of the four stores of a chunk, in the first tile
#pragma unroll
    for (int y = 0; y < 4; ++y) to[y] = smem_u32(sKV) + row0 * 128 + (((chunk0 * 4 + y) ^ (row0 & 7)) << 4);
    uint32_t ring = 0, used = 0, block = 0, part = 0, looks = 0; // part: number of the segment
    Seg s;
    while (!failed && walk.next(s)) {
      const int halves = 2 * (s.j1 - s.j0);
      float k_by = 1.f, v_by = 1.f;
#pragma unroll 1
      for (int i = 0; i < halves; ++i) {                        // K and V in turn
        const uint32_t stage = used % L::AHEAD, st = ring % L::STAGES;
        if (!__all_sync(0xffffffffu, mma_wait(bar_code_full + 8 * stage, (used / L::AHEAD) & 1))) { failed = true; break; }
        const int left = s.len - (s.j0 + (i >> 1)) * 128;        // rows of the sequence from this block on
        const uint32_t slot = (block + (i >> 1)) % CK_FLAGS;
        uint4 code[CH];
        uint32_t par[CH];
        bool any = false, close = false;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
          code[k] = lds128(code0 + stage * L::STAGED + (row_of(k) - row0) * L::PITCH + (chunk_of(k) - chunk0) * 16);
          par[k] = lds32(par0 + stage * L::STAGED + ((row_of(k) - row0) * NG + chunk_of(k) * 32 / G) * 4);
        }
        if (left < 128) {                                        // behind the sequence: zeros, whatever lies there
#pragma unroll
          for (int k = 0; k < CH; ++k) {
            if (row_of(k) >= left) {
              code[k] = make_uint4(0, 0, 0, 0);
              par[k] = 0;
            }
          }
        }
        // lo below 2^15 and scale below 2^11 in size: all values fit; else a closer look
#pragma unroll
        for (int k = 0; k < CH; ++k) close |= (par[k] << 17) >= 0x47000000u << 1 || (par[k] & 0x7fff0000u) >= 0x45000000u;
        if (__any_sync(0xffffffffu, close)) {
          uint32_t* notes = s_notes + slot * 16 + (warp & 3);
          if ((i & 1) && lane < 4) notes[lane * 4] = 0;
          __syncwarp();
#pragma unroll 1
          for (int k = 0; k < CH; ++k) {
            uint32_t pp = par[0];
#pragma unroll
            for (int x = 1; x < CH; ++x) pp = k == x ? par[x] : pp;
            const bool bad = !fits_half(pp, p.status);
            any |= bad;
            if (bad && (i & 1)) atomicOr(notes + chunk_of(k) * 32 / G * 4, 1u << (row_of(k) & 31));
            // a key becomes NaN, and so do the scores of who sees it; a value zero
#pragma unroll
            for (int x = 0; x < CH; ++x)
              if (k == x && bad) par[x] = i & 1 ? 0u : 0x7fc07fc0u;
          }
          any = __any_sync(0xffffffffu, any);
        }
        if (i < 2) {                                             // the part's first keys and values: their unit
          bool ordinary = false;
#pragma unroll
          for (int k = 0; k < CH; ++k) ordinary |= !is_small(size_of(par[k]));
          uint32_t u = 0;
          if (left > (warp & 3) * 32 && !__any_sync(0xffffffffu, ordinary))
            u = unit_of_part<D, G>(p, i ? p.v_params : p.k_params, smem_u32(s_staging) + stage * L::STAGED + L::CODES, s_sizes, bar_sizes, &looks, s.b, s.h, s.j0, s.j1, s.len,
                                   warp & 3, lane);
          if (u == NO_UNIT) { failed = true; break; }
          if (warp == 8 && lane == 0) reinterpret_cast<uint8_t*>(s_units + part % CK_FLAGS)[i] = static_cast<uint8_t>(u);
          if (i) v_by = exp2_of(static_cast<int>(u));
          else k_by = exp2_of(static_cast<int>(u));
        }
        // (A bulk copy may overwrite what was read only behind a fence between the two kinds of access: without it, calls in close succession
        // found codes of a later block in a tile's second half.)
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_code_empty + 8 * stage);
        if (!__all_sync(0xffffffffu, mma_wait(bar_kv_empty + 8 * st, ((ring / L::STAGES) & 1) ^ 1))) { failed = true; break; }
        ++used;
        ++ring;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
          const uint32_t word[4] = {code[k].x, code[k].y, code[k].z, code[k].w};
          const Params16 x = params16(par[k], i & 1 ? v_by : k_by);
          // a nibble in the low bits of a number from 1024 on, or four bits up in one from 64 on: that plus the code; then the code
          // times scale plus lo in one rounding
          const __half2 m1024 = half2_of(0xe400e400u), m64 = half2_of(0xd400d400u), lo2 = half2_of(x.lo2), sc2 = half2_of(x.scale2);
          // (16 rows down: the same place of the swizzle; at width 96 the second chunk of a pair is four 16-byte places away)
          const uint32_t tile = st * L::TILE + (D == 96 ? 0 : (k & 1) * 16 * 128) + (k >> 1) * L::SUB, flip = D == 96 ? (k & 1) * 64 : 0;
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t n = e ? word[y] >> 8 : word[y];
              const __half2 a = __hfma2(__hadd2(half2_of((n & 0x000f000fu) | 0x64006400u), m1024), sc2, lo2);
              const __half2 b = __hfma2(__hadd2(half2_of((n & 0x00f000f0u) | 0x54005400u), m64), sc2, lo2);
              w[2 * e] = *reinterpret_cast<const uint32_t*>(&a);
              w[2 * e + 1] = *reinterpret_cast<const uint32_t*>(&b);
            }
            sts128((to[y] ^ flip) + tile, w[0], w[1], w[2], w[3]);
          }
        }
        if ((i & 1) && lane == 0) reinterpret_cast<uint8_t*>(s_any + slot)[warp & 3] = any;
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_kv_full + 8 * st);
      }
      block += s.j1 - s.j0;
      ++part;
    }
    if (failed && lane == 0) report(p.status, DEV_TIMEOUT_PRODUCER);
  } else {
    if (warp < 14) {
      // ------------------------------------------------------------------ MMA issuers, one per tile
      const int t = warp - 12;
      const uint32_t idesc_s = make_idesc(ACC_F32, FMT_F16, FMT_F16, 128, 64);
      const uint32_t idesc_o = make_idesc(ACC_F32, FMT_F16, FMT_F16, 128, D, 0, 1);
      const uint32_t d_s = tmem_base + t * 128, d_o = tmem_base + 256 + t * 128;
      const uint32_t q0_lo = desc_lo(smem_u32(sQ), 16), k_lo = desc_lo(smem_u32(sKV), 16), v_lo = desc_lo(smem_u32(sKV), L::SUB);
      const uint32_t s_full = bar_s_full + 16 * t, p_full = bar_p_full + 16 * t, o_full = bar_o_full + 16 * t;
      uint32_t ring = 0, qn = 0, pn = 0;
      Seg s;
      while (walk.next(s)) {
        if (lane == 0) {
          const bool twin = s.twin();
          const int blocks = s.j1 - s.j0, n = twin ? (blocks + 1 - t) >> 1 : blocks;        // mine
          const uint32_t step = twin ? 4 : 2, first = ring + (twin ? 2 * t : 0);            // K of my block i: first + step i
          const uint32_t q_lo = q0_lo + (twin ? 0u : t * (L::TILE >> 4));
          auto kv_ready = [&](uint32_t pos) { return mma_wait(bar_kv_full + 8 * (pos % L::STAGES), (pos / L::STAGES) & 1); };
          // (what only one tile uses is given back by it alone, twice over)
          auto kv_done = [&](uint32_t pos) {
            const uint32_t bar = bar_kv_empty + 8 * (pos % L::STAGES);
            if (twin) mbar_arrive(bar);
            umma_commit(bar);
          };
          auto kv_there = [&](uint32_t pos) { return mbar_test(bar_kv_full + 8 * (pos % L::STAGES), (pos / L::STAGES) & 1); };
          bool late = false;                                     // the first half's next scores are still to be issued
          // S of keys 64 h .. 64 h + 63 of the block at ring position `pos`
          auto scores = [&](uint32_t pos, int h) {
            const uint32_t kb = k_lo + (pos % L::STAGES) * (L::TILE >> 4) + h * (64 * 128 >> 4);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              const uint32_t off = ((k >> 2) * L::SUB + (k & 3) * 32) >> 4;
              if (k == 0) mma_ss<false>(d_s + h * 64, q_lo + off, kb + off, idesc_s);
              else mma_ss<true>(d_s + h * 64, q_lo + off, kb + off, idesc_s);
            }
            umma_commit(s_full + 8 * h);
          };
          // Also a tile without blocks of its own waits for Q, so that no issuer gets more than a segment ahead.
          failed = !mma_wait(bar_q_full, qn++ & 1);
          if (n == 0) mbar_arrive(bar_q_empty);
          // Batch x: O += P V of my half block x, then S of the second next one, which takes its place; the first two have only scores.
#pragma unroll 1
          for (int x = -2; x < 2 * n && !failed; ++x) {
            const int h = x & 1, i = x >> 1;
            const uint32_t vpos = first + step * i + 1, kpos = first + step * (i + 1);
            if (x >= 0) {
              if ((h == 0 && !kv_ready(vpos)) || !mma_wait(p_full + 8 * h, pn & 1)) { failed = true; break; }
              tc_fence_after();
              const uint32_t vb = v_lo + (vpos % L::STAGES) * (L::TILE >> 4) + h * 512;
#pragma unroll
              for (int k = 0; k < 4; ++k) mma_ts(d_o, d_s + h * 64 + k * 8, vb + k * 128, idesc_o, k || x);
              umma_commit(o_full + 8 * h);
              if (h) kv_done(vpos);
              pn += h;
            }
            if (x + 2 < 2 * n) {
              // Keys that are not there yet must not hold up the product with the second half's probabilities, which gives back the place
              // of the values that are to be widened before those keys.
              if (h == 0) {
                late = x >= 0 && !kv_there(kpos);
                if (late) continue;
              }
              if ((h == 0 || late) && !kv_ready(kpos)) { failed = true; break; }
              // These scores overwrite the probabilities that the product just issued reads, and products into unlike accumulators are
              // promised no order: it has to be complete.  (The softmax works on the other half meanwhile.)
              if (x >= 0 && !((h == 0 || late ? mma_wait(o_full, (pn - h) & 1) : true) && (h == 1 ? mma_wait(o_full + 8, (pn - 1) & 1) : true))) { failed = true; break; }
              tc_fence_after();
              if (late) scores(kpos, 0);
              scores(kpos, h);
              if (h) kv_done(kpos);
              if (x + 3 == 2 * n) umma_commit(bar_q_empty);
            }
          }
          ring += 2 * blocks;
          if (failed) report(p.status, DEV_TIMEOUT_MMA);
        }
        if (__any_sync(0xffffffffu, failed)) { failed = true; break; }
      }
    } else if (warp == 14) {
      // ------------------------------------------------------------------ what is left to the joining kernel
      Note note = {};
      Seg s;
      while (walk.next(s)) {
        if (s.j0 > 0) note.ends = s.j1 == s.n;
        else if (s.j1 < s.n) {
          note.rows = s.rows;
          note.q0 = s.q0;
          note.row0 = s.row0;
          note.h = s.h;
        }
      }
      if (lane == 0) space.note[me] = note;
    } else {
      // ------------------------------------------------------------------ codes and parameters on their way
      const int piece_shift = min(p.page_shift, 7), pieces = 128 >> piece_shift, piece = 1 << piece_shift;      // of a block's rows in one page
      uint32_t filled = 0;
      Seg s;
      while (!failed && walk.next(s)) {
        const int* table = p.table + s.b * p.table_stride;
        // the page that has my piece of block j (the lanes of a block's pieces), and the next block's on its way
        auto page_of = [&](int j) {
          const int t = j * 128 + lane * piece;
          return lane < pieces && j < s.j1 && t < s.len ? table[t >> p.page_shift] : 0;
        };
        // Staging holds a block and a half, not enough to cover the memory's latency: what follows is called into the L2 before.
        auto fetch = [&](int j, int page) {
          const int t = j * 128 + lane * piece;
          if (lane >= pieces || j >= s.j1 || t >= s.len || page < 0 || page >= p.num_pages) return;
          const int64_t at = ((static_cast<int64_t>(page) * p.Hk + s.h) << p.page_shift) + (t & ((1 << p.page_shift) - 1));
          bulk_prefetch(p.k_codes + at * L::PITCH, piece * L::PITCH);
          bulk_prefetch(p.v_codes + at * L::PITCH, piece * L::PITCH);
          bulk_prefetch(p.k_params + at * NG, piece * (NG * 4));
          bulk_prefetch(p.v_params + at * NG, piece * (NG * 4));
        };
#pragma unroll 1
        for (int j = s.j0 + 1; j < min(s.j0 + CK_FETCH, s.j1); ++j) fetch(j, page_of(j));
        int next = page_of(s.j0), far = page_of(s.j0 + CK_FETCH);
#pragma unroll 1
        for (int j = s.j0; j < s.j1 && !failed; ++j) {
          int page = next;
          fetch(j + CK_FETCH, far);
          next = page_of(j + 1);
          far = page_of(j + 1 + CK_FETCH);
          if (page < 0 || page >= p.num_pages) {
            report(p.status, DEV_BAD_PAGE);
            page = 0;
          }
          const int t = j * 128 + lane * piece;
          const bool copies = lane < pieces && t < s.len;
          const int64_t at = ((static_cast<int64_t>(page) * p.Hk + s.h) << p.page_shift) + (t & ((1 << p.page_shift) - 1));
          const uint32_t count = static_cast<uint32_t>(min(pieces, max(0, (s.len - j * 128 + piece - 1) >> piece_shift)));
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            const uint32_t stage = filled % L::AHEAD, bar = bar_code_full + 8 * stage, to = smem_u32(s_staging) + stage * L::STAGED;
            if (!mma_wait(bar_code_empty + 8 * stage, ((filled / L::AHEAD) & 1) ^ 1)) failed = true;
            if (__any_sync(0xffffffffu, failed)) { failed = true; break; }
            ++filled;
            if (lane == 0) mbar_arrive_expect_tx(bar, count * (piece * static_cast<uint32_t>(L::PITCH + NG * 4)));
            __syncwarp();
            if (copies) {
              bulk_load(to + lane * piece * L::PITCH, (v ? p.v_codes : p.k_codes) + at * L::PITCH, piece * L::PITCH, bar);
              bulk_load(to + L::CODES + lane * piece * (NG * 4), (v ? p.v_params : p.k_params) + at * NG, piece * (NG * 4), bar);
            }
          }
        }
      }
      if (failed && lane == 0) report(p.status, DEV_TIMEOUT_PRODUCER);
    }
  }
  if (failed) {                                                  // products in flight come to rest before the block exits
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) {
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 12) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

// Joins the pieces of an item that begins in one CTA without ending there: that CTA's second piece, and the following ones' first.  A block
// has 32 rows and 32 columns: two warps of 16 columns, for each of them WAYS that take every WAYS-th piece and are then joined
// in shared memory, all in a fixed order.  (With one thread for all pieces of a row, an item in 74 pieces took 115 us.)
//   FEW    eight warps a column and a block for each item there can be, which looks it up in all notes: where items have eight
//          pieces and more (48 tokens at the end of 60000: 42 us for the call instead of 46)
//   else   four, and a block for every CTA, which looks at the item that begins there (many items: 176 us for the batch of 32 sequences,
//          182 with eight warps; 188 looking items up)
template <int D, bool FEW>
__global__ void __launch_bounds__(FEW ? 512 : 256) attn_chunk_join_kernel(const __grid_constant__ ChunkParams p, const int ctas) {
  constexpr int WAYS = FEW ? 8 : 4;
  __shared__ float4 s_o[WAYS][2][4][32];
  __shared__ float2 s_ml[WAYS][2][32];
  wait_for_predecessor();
  const ChunkSpace<D> space(p.ws, ctas);
  const int lane = threadIdx.x & 31, way = threadIdx.x >> 6, half = threadIdx.x >> 5 & 1;
  const int row = blockIdx.y * 32 + lane, col = blockIdx.z * 32 + half * 16;
  int c0 = blockIdx.x, n = 1;                                    // pieces: up to the first that reaches the item's end
  if constexpr (FEW) {
    int skip = blockIdx.x, end = ctas;
    c0 = -1;
#pragma unroll 5
    for (int c = 0; c < ctas; c += 32) {
      const bool in = c + lane < ctas;
      const int rows = in ? space.note[c + lane].rows : 0, ends = in ? space.note[c + lane].ends : 0;
      const uint32_t begin = __ballot_sync(0xffffffffu, rows > 0);
      uint32_t ending = __ballot_sync(0xffffffffu, ends);
      if (c0 < 0) {
        const uint32_t here = __ballot_sync(0xffffffffu, rows > 0 && __popc(begin & ((1u << lane) - 1)) == skip);
        skip -= __popc(begin);
        if (!here) continue;
        c0 = c + __ffs(here) - 1;
        ending &= ~(here | (here - 1));
      }
      if (ending && end == ctas) end = c + __ffs(ending);
    }
    if (c0 < 0) return;
    n = end - c0;
  }
  const Note note = space.note[c0];
  if (static_cast<int>(blockIdx.y) * 32 >= note.rows) return;
  if constexpr (!FEW) {
    for (int c = c0 + 1;; c += 32) {
      const uint32_t end = __ballot_sync(0xffffffffu, c + lane >= ctas || space.note[c + lane].ends);
      n += end ? __ffs(end) : 32;
      if (end) break;
    }
    n = min(n, ctas - c0);
  }
  float m = -INFINITY, l = 0.f;
  float4 a[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) a[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
  for (int i = way; i < n; i += WAYS) {
    const int64_t piece = 2 * static_cast<int64_t>(c0 + i) + (i == 0);
    const float2 x = space.ml[piece * CK_ROWS + row];
    float4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = space.o[(piece * (D / 4) + col / 4 + k) * CK_ROWS + row];
    const float mn = fmaxf(m, x.x), ref = mn == -INFINITY ? 0.f : mn;
    const float f = ap_ex2(m - ref), g = ap_ex2(x.x - ref);      // 0 for what saw nothing; NaN sums pass
    m = mn;
    l = fmaf(l, f, x.y * g);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      a[k].x = fmaf(a[k].x, f, v[k].x * g);
      a[k].y = fmaf(a[k].y, f, v[k].y * g);
      a[k].z = fmaf(a[k].z, f, v[k].z * g);
      a[k].w = fmaf(a[k].w, f, v[k].w * g);
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) s_o[way][half][k][lane] = a[k];
  s_ml[way][half][lane] = make_float2(m, l);
  __syncthreads();
  if (way != 0 || row >= note.rows) return;
#pragma unroll
  for (int w = 1; w < WAYS; ++w) {
    const float2 x = s_ml[w][half][lane];
    const float mn = fmaxf(m, x.x), ref = mn == -INFINITY ? 0.f : mn;
    const float f = ap_ex2(m - ref), g = ap_ex2(x.x - ref);
    m = mn;
    l = fmaf(l, f, x.y * g);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 v = s_o[w][half][k][lane];
      a[k].x = fmaf(a[k].x, f, v.x * g);
      a[k].y = fmaf(a[k].y, f, v.y * g);
      a[k].z = fmaf(a[k].z, f, v.z * g);
      a[k].w = fmaf(a[k].w, f, v.w * g);
    }
  }
  const float r = l == 0.f ? 0.f : 1.0f / l;
  const int my_row = note.row0 + row, token = my_row / p.g;
  uint4* dst = reinterpret_cast<uint4*>(p.o + static_cast<int64_t>(note.q0 + token) * p.o_tok + static_cast<int64_t>(note.h * p.g + my_row - token * p.g) * p.o_head + col);
#pragma unroll
  for (int k = 0; k < 2; ++k)
    dst[k] = make_uint4(ap_pack(a[2 * k].x * r, a[2 * k].y * r), ap_pack(a[2 * k].z * r, a[2 * k].w * r), ap_pack(a[2 * k + 1].x * r, a[2 * k + 1].y * r),
                        ap_pack(a[2 * k + 1].z * r, a[2 * k + 1].w * r));
}

namespace {
template <int D, int G, typename List>
cudaError_t run(const ChunkParams& p, int ctas, cudaStream_t s) {
  auto kern = attn_chunk_kernel<D, G, List>;
  cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), (ChunkLayout<D, G>::SMEM));
  if (e != cudaSuccess) return e;
  if (!std::is_same<List, ListShared>::value) {
    e = launch_following(attn_chunk_list_kernel<D>, dim3(1), CK_THREADS, 0, s, p, ctas);
    if (e != cudaSuccess) return e;
  }
  e = launch_following(kern, dim3(static_cast<unsigned>(ctas)), CK_THREADS, (ChunkLayout<D, G>::SMEM), s, p);
  if (e != cudaSuccess || ctas == 1) return e;
  const int64_t items = static_cast<int64_t>(p.most_items) * p.Hk;
  const unsigned rows = static_cast<unsigned>((p.q_tokens * p.g < CK_ROWS ? p.q_tokens * p.g + 31 : CK_ROWS) / 32);
  if (items * 8 <= ctas) return launch_following(attn_chunk_join_kernel<D, true>, dim3(static_cast<unsigned>(items), rows, D / 32), 512, 0, s, p, ctas);
  return launch_following(attn_chunk_join_kernel<D, false>, dim3(static_cast<unsigned>(ctas), rows, D / 32), 256, 0, s, p, ctas);
}
template <int D, int G>
cudaError_t by_list(const ChunkParams& p, int ctas, cudaStream_t s) {
  return p.most_items <= CK_MAX_LIST ? run<D, G, ListShared>(p, ctas, s) : run<D, G, ListGlobal>(p, ctas, s);
}
template <int D>
size_t space_bytes(int ctas, int64_t most_items) {
  return static_cast<size_t>(ctas) * (2 * CK_ROWS * (D * 4 + 8) + sizeof(Note)) + (most_items > CK_MAX_LIST ? (most_items + 1) * sizeof(int4) : 0);
}
}  // namespace

// Items per head there can be at most (a sequence's last one may be short), and CTAs for them: one an SM, or one for every
// CK_LEAST units there can be where that is fewer.
int64_t attn_chunk_items(int64_t q_tokens, int B, int g) { return q_tokens * g / CK_ROWS + B; }
int attn_chunk_ctas(int64_t items, int Hk, int max_len, int num_sms) {
  const int64_t units = items * Hk * (((max_len + 127) / 128 + 1) * CK_BLOCK + CK_START), want = units / CK_LEAST + 1;
  return static_cast<int>(want < num_sms ? want : num_sms);
}
size_t attn_chunk_bytes(int D, int ctas, int64_t most_items) {
  return D == 64 ? space_bytes<64>(ctas, most_items) : D == 96 ? space_bytes<96>(ctas, most_items) : space_bytes<128>(ctas, most_items);
}

cudaError_t launch_attn_chunk(const ChunkParams& p, int D, int G, int ctas, cudaStream_t s) {
  if (D == 64) return G == 32 ? by_list<64, 32>(p, ctas, s) : by_list<64, 64>(p, ctas, s);
  if (D == 96) return by_list<96, 32>(p, ctas, s);
  return G == 32 ? by_list<128, 32>(p, ctas, s) : G == 64 ? by_list<128, 64>(p, ctas, s) : by_list<128, 128>(p, ctas, s);
}

}  // namespace gc
