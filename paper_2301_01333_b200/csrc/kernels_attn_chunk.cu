// Attention of chunks of new tokens over the paged 4-bit cache: any number of query rows per sequence, packed one behind the other.
//
//   O = softmax(scale Q K^T) V, blockwise over 128 keys with a running reference, as in the prompt attention, K, V = lo + code * scale
//
// The products are tcgen05's with fp32 accumulators and fp16 operands: K, V and the probabilities are rounded once, to eleven bits.  (In bf16 the
// rounding of K alone puts the output off by 3-5e-3 of its norm, which is mostly cancellation, where the output's own rounding is 1.7e-3.)  Q, bf16,
// becomes fp16 exactly after its row is scaled by a power of two; probabilities, at most 2^4 relative to the reference, are lifted by 2^11.
//
// A row is a (token, query head) of those that share a key/value head, token by token, so that a block of keys, once widened, serves
// all of them.  A CTA holds 256 rows in two tiles of 128, and per block of 128 keys at width 128 there are
// two products of 512 clocks for each tile (2048 in all), as many clocks of exponentials (16 a clock), and 32768 elements to be
// widened: 3.4 instructions for two of them, 440 of the 2048 issue slots of a scheduler.
//   warps 0-3, 4-7   softmax of tile 0 / 1, one row per thread (as in the prompt attention)
//   warps 8-11       widen: a thread per key row; codes come from global memory into registers a block ahead, and go as fp16 into
//                    128-byte-swizzled tiles of a ring, where a thread's row makes the store free of bank conflicts.  The eight elements of a word come
//                    apart as (0,4), (1,5), (2,6), (3,7) and stay in that order: Q's elements are put in the same one, and
//                    the columns of O are put back in registers at the end.
//   warps 12, 13     MMA issuers of tile 0 / 1, taking turns
//   warp 14          notes down which pieces of split items this CTA leaves
// Where an item has at most 128 rows the two tiles are the same rows: they take the even and the odd blocks of keys, and
// are joined at the end, the one reading the other's O from tensor memory.
// The work is a row of units (one block of keys of one item; an item is 256 rows of a sequence, times heads), of which every CTA
// takes an equal stretch; the pieces of an item that stretches cut are joined in their order by a second kernel.
//   * A value that is not finite must not reach rows that do not see it (0 times NaN): such groups are widened as zeros and
//     noted in a bit mask per block; a row that does see one gets NaN in that group's columns.
#include <cuda_fp16.h>

#include <atomic>

#include "attn_tc.cuh"
#include "ptx.cuh"
#include "serving.cuh"

namespace gc {

namespace {
constexpr int CK_THREADS = 512, CK_ROWS = 256;
constexpr int CK_MAX_LIST = 1024;            // items per head that are listed in shared memory
constexpr int CK_FLAGS = 8;                  // blocks whose notes of values that are not finite are kept
constexpr float CK_RAISE = 4.0f;             // binades a score may exceed the reference by
constexpr float CK_LIFT = 11.0f;             // binades the probabilities are lifted by: at most 2^15, and whole down to 2^-25 of the reference
constexpr float CK_LARGEST = 65504.0f;       // the largest fp16
// Registers a thread: what the kernel has to be compiled to, and the warpgroups' shares of them (kernels_attn_prompt.cu has the reason).
constexpr int CK_REGS = 128, CK_REGS_SOFTMAX = 192, CK_REGS_WIDEN = 72, CK_REGS_MMA = 56;
static_assert(2 * CK_REGS_SOFTMAX + CK_REGS_WIDEN + CK_REGS_MMA <= 4 * CK_REGS, "the warpgroups' shares exceed the launch's registers");

template <int D>
struct ChunkLayout {
  static constexpr int NSUB = (D + 63) / 64;     // 64-element sub-tiles of 128-byte rows
  static constexpr int SUB = 128 * 128;
  static constexpr int TILE = NSUB * SUB;        // 128 rows of Q, K or V
  static constexpr int STAGES = D == 64 ? 8 : 4;
  static constexpr int BARS = 2 * STAGES + 14;
  // Q, ring, list, notes [CK_FLAGS][4 groups][4 words], one word a block that sums them up, sums of the second tile [3][128], factors
  // of the rows [2][256]
  static constexpr int LIST = CK_MAX_LIST * 8, NOTES = CK_FLAGS * 16 * 4, ANY = CK_FLAGS * 4, SUMS = 3 * 128 * 4, FACTORS = 2 * CK_ROWS * 4;
  static constexpr size_t SMEM = 1024 + static_cast<size_t>(2 + STAGES) * TILE + LIST + NOTES + ANY + SUMS + FACTORS + BARS * 8 + 64 * 4;
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
  if (fmaxf(fabsf(lo), fabsf(fmaf(15.f, scale, lo))) <= CK_LARGEST && fabsf(scale) <= CK_LARGEST) return true;      // (the first holds for a NaN too)
  if (fabsf(lo) < INFINITY && fabsf(scale) < INFINITY) report(status, DEV_LARGE_HALF);
  return false;
}
__device__ __forceinline__ Params16 params16(uint32_t par) {
  const uint32_t lo = pack_half(__uint_as_float(par << 16), __uint_as_float(par << 16));
  const uint32_t scale = pack_half(__uint_as_float(par & 0xffff0000u), __uint_as_float(par & 0xffff0000u));
  return Params16{lo, scale};
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
template <typename List>
__device__ int2 make_list(const ChunkParams& p, const List& list, int most, int* s_sums, int* s_first) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int items = 0;
  for (int s0 = 0; s0 < p.B; s0 += CK_THREADS) {
    const int b = s0 + tid;
    int count = 0;
    if (b < p.B) {
      const ChunkSeq s = seq_of(p, b);
      count = items_of(p, s);
      if (blockIdx.x == 0) {
        if (p.cu_q[b] != s.q0 || p.cu_q[b + 1] != s.q0 + s.nq) report(p.status, DEV_BAD_OFFSETS);
        if (p.lengths[b] != s.len) report(p.status, DEV_BAD_LENGTH);
      }
    }
    int all;
    const int before = block_scan(count, s_sums, &all);
    s_first[tid] = items + before;
    __syncthreads();
    for (int w = warp; w < CK_THREADS && s0 + w < p.B; w += CK_THREADS / 32) {
      const ChunkSeq s = seq_of(p, s0 + w);
      const int n = items_of(p, s), first = s_first[w];
      for (int i = lane; i < n && first + i < most; i += 32) list.put(first + i, blocks_of(p, s, i), s0 + w, i);
    }
    items = min(items + all, most);
    __syncthreads();
  }
  int units = 0;
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

// Where CTA number c's stretch begins.
__device__ __forceinline__ int64_t cut(int64_t total, int c, int ctas) { return total / ctas * c + min(static_cast<int64_t>(c), total % ctas); }

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
    h = static_cast<int>(from / units);
    const int at = static_cast<int>(from - static_cast<int64_t>(h) * units);
    int lo = 0, hi = items - 1;                                  // the last item that does not begin behind `at`
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (list.get(mid).before <= at) lo = mid;
      else hi = mid - 1;
    }
    e = lo;
    j = at - list.get(e).before;
  }
  __device__ __forceinline__ bool next(Seg& s) {
    if (left <= 0) return false;
    const Entry x = list.get(e);
    const ChunkSeq q = seq_of(p, x.b);
    s.b = x.b;
    s.h = h;
    s.row0 = x.i * CK_ROWS;
    s.rows = min(q.nq * p.g - s.row0, CK_ROWS);
    s.q0 = q.q0;
    s.len = q.len;
    s.ahead = q.len - q.nq;
    s.n = blocks_of(p, q, x.i);
    s.j0 = j;
    s.j1 = static_cast<int>(min(static_cast<int64_t>(s.n), j + left));
    left -= s.j1 - s.j0;
    j = 0;
    if (++e == items) {
      e = 0;
      ++h;
    }
    return true;
  }
};

// What a CTA leaves to the joining kernel: a piece that begins an item without reaching its end (slot 1; rows > 0), and one that
// begins inside an item (slot 0), which may reach its end.
struct Note {
  int rows, q0, row0, h;
  int ends, pad[3];
};
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
  __shared__ int s_sums[CK_THREADS / 32], s_first[CK_THREADS];
  wait_for_predecessor();
  int4* list = ChunkSpace<D>(p.ws, ctas).list;
  const int2 got = make_list(p, ListGlobal{list + 1}, p.most_items, s_sums, s_first);
  if (threadIdx.x == 0) list[0] = make_int4(got.x, got.y, 0, 0);
}

template <int D, int G, typename List>
__global__ void __launch_bounds__(CK_THREADS, 1) attn_chunk_kernel(const __grid_constant__ ChunkParams p) {
  using L = ChunkLayout<D>;
  constexpr int NG = D / G;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = smem;                                           // [2] tiles
  uint8_t* sKV = sQ + 2 * L::TILE;                              // [STAGES] tiles
  uint2* s_list = reinterpret_cast<uint2*>(sKV + L::STAGES * L::TILE);
  uint32_t* s_notes = reinterpret_cast<uint32_t*>(s_list + CK_MAX_LIST);        // [CK_FLAGS][4][4]
  uint32_t* s_any = s_notes + CK_FLAGS * 16;                    // [CK_FLAGS], a byte per widening warp
  float* s_second = reinterpret_cast<float*>(s_any + CK_FLAGS); // reference, sum and groups that are not finite of tile 1
  float* s_factor = s_second + 3 * 128;                         // [2 segments][256]: c times the power of two a row's scores are short of
  uint64_t* bars = reinterpret_cast<uint64_t*>(s_factor + 2 * CK_ROWS);
  const uint32_t b0 = smem_u32(bars);
  const uint32_t bar_q_full = b0, bar_q_empty = b0 + 8, bar_s_full = b0 + 16, bar_p_full = b0 + 32, bar_o_full = b0 + 64;
  const uint32_t bar_turn = b0 + 80, bar_second = b0 + 96, bar_joined = b0 + 104, bar_kv_full = b0 + 112, bar_kv_empty = bar_kv_full + 8 * L::STAGES;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + L::BARS);
  int* s_sums = reinterpret_cast<int*>(tmem_slot + 4);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    mbar_init(bar_q_full, 4);
    mbar_init(bar_q_empty, 2);                                  // both tiles' issuers
    mbar_init(bar_second, 4);
    mbar_init(bar_joined, 4);
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_s_full + 8 * i, 1);
      mbar_init(bar_o_full + 8 * i, 1);
      mbar_init(bar_turn + 8 * i, 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(bar_p_full + 8 * i, 4);
    for (int i = 0; i < L::STAGES; ++i) {
      mbar_init(bar_kv_full + 8 * i, 4);
      mbar_init(bar_kv_empty + 8 * i, 2);
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
    size = make_list(p, list, CK_MAX_LIST, s_sums, reinterpret_cast<int*>(sQ));
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
  // Stretches of at least p.least units: fewer CTAs work where there is little to do.
  const int64_t total = static_cast<int64_t>(size.y) * p.Hk;
  const int working = static_cast<int>(min(static_cast<int64_t>(ctas), max((total + p.least - 1) / p.least, static_cast<int64_t>(1))));
  const int me = static_cast<int>(blockIdx.x);
  Walk<List> walk(p, list, size.x, size.y, me < working ? cut(total, me, working) : 0, me < working ? cut(total, me + 1, working) : 0);

  bool failed = false;
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(CK_REGS_SOFTMAX));
    // ------------------------------------------------------------------ softmax and output
    const int t = warp >> 2, row = tid & 127;
    const uint32_t t_lane = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t s_addr = t_lane + t * 128, o_addr = t_lane + 256 + t * 128;
    uint32_t sn = 0, on = 0, jn = 0, block = 0;                 // block: number of the segment's first among all of this CTA's
    Seg s;
    for (uint32_t seg = 0; !failed && walk.next(s); ++seg) {
      const bool twin = s.twin();
      const int my_row = s.row0 + (twin ? row : t * 128 + row);
      const bool mine = my_row < s.row0 + s.rows;
      const int token = mine ? my_row / p.g : 0;
      const int lim = mine ? max(min(s.ahead + token + 1, s.len), 0) : 0;
      const int j_first = twin ? s.j0 + t : s.j0, j_step = twin ? 2 : 1;
      float m = -INFINITY, l = 0.f, c = 0.f;
      uint32_t poison = 0;                                      // groups of columns in which this row saw a value that is not finite
      int seen_blocks = 0;
      for (int j = j_first; j < s.j1; j += j_step) {
        if (!__all_sync(0xffffffffu, mbar_wait(bar_s_full + 8 * t, sn & 1))) { failed = true; break; }
        ++sn;
        tc_fence_after();
        uint32_t v[2][64];
        if (j == j_first) c = s_factor[(seg & 1) * CK_ROWS + (twin ? row : t * 128 + row)];
        tmem_ld64(s_addr, v[0]);
        tmem_ld64(s_addr + 64, v[1]);
        const int left = lim - j * 128;
        {
          // (written before this block's keys were handed over, and not again before all rows have handed over their probabilities)
          const uint32_t slot = (block + j - s.j0) % CK_FLAGS;
          if (s_any[slot]) {
#pragma unroll
            for (int g = 0; g < NG; ++g) {
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                const int k = left - 32 * w;
                const uint32_t sees = k >= 32 ? 0xffffffffu : k <= 0 ? 0u : (1u << k) - 1u;
                if (s_notes[slot * 16 + g * 4 + w] & sees) poison |= 1u << g;
              }
            }
          }
        }
        if (__any_sync(0xffffffffu, left < 128)) {
#pragma unroll
          for (int i = 0; i < 128; ++i)
            if (i >= left) v[i >> 6][i & 63] = 0xff800000u;      // minus infinity, whatever the score was
        }
        float top[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) top[i] = max3(__uint_as_float(v[i >> 1][(i & 1) * 32]), __uint_as_float(v[i >> 1][(i & 1) * 32 + 1]), -INFINITY);
#pragma unroll
        for (int i = 2; i < 32; i += 2) {
#pragma unroll
          for (int k = 0; k < 4; ++k) top[k] = max3(top[k], __uint_as_float(v[k >> 1][(k & 1) * 32 + i]), __uint_as_float(v[k >> 1][(k & 1) * 32 + i + 1]));
        }
        const float mx = max3(max3(top[0], top[1], top[2]), top[3], top[3]);
        if (__any_sync(0xffffffffu, (mx - m) * c > CK_RAISE)) {
          const float mn = fmaxf(m, mx);
          if (score_too_large(mn * c)) report(p.status, DEV_LARGE_SCORE);
          const float f = mn == m ? 1.f : ap_ex2((m - mn) * c);  // 0 from the initial minus infinity
          m = mn;
          l *= f;
          if (seen_blocks > 0) {
            // S of this block is complete, hence so is the product of the block before: O is at rest
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
        ++seen_blocks;
        const float off = m == -INFINITY ? 0.f : fmaf(-m, c, CK_LIFT);
        const uint64_t c2 = pair2(c, c), off2 = pair2(off, off);
        uint64_t ls[2] = {0, 0};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t w[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            float e0, e1;
            unpair2(fma2(pair2(__uint_as_float(v[h][2 * i]), __uint_as_float(v[h][2 * i + 1])), c2, off2), &e0, &e1);
            e0 = ap_ex2(e0);
            e1 = ap_ex2(e1);
            ls[i & 1] = add2(ls[i & 1], pair2(e0, e1));
            w[i] = pack_half(e0, e1);
          }
          tmem_st32(s_addr + h * 32, w);
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_p_full + 8 * (2 * t + h));
        }
        float l0, l1;
        unpair2(add2(ls[0], ls[1]), &l0, &l1);
        l += l0 + l1;
      }
      if (failed) break;
      block += s.j1 - s.j0;
      if (seen_blocks) {
        if (!__all_sync(0xffffffffu, mbar_wait(bar_o_full + 8 * t, on & 1))) { failed = true; break; }
        ++on;
        tc_fence_after();
      }
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
        if (!__all_sync(0xffffffffu, mbar_wait(bar_joined, jn & 1))) { failed = true; break; }
        ++jn;
        tc_fence_after();
        continue;
      }
      if (twin) {
        if (!__all_sync(0xffffffffu, mbar_wait(bar_second, jn & 1))) { failed = true; break; }
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
      const bool whole = s.whole();
      const float rl = l == 0.f ? 0.f : whole ? 1.0f / l : 1.f;
      const float a0 = f0 * rl, a1 = f1 * rl;
      const int64_t piece = 2 * static_cast<int64_t>(me) + (s.j0 == 0);
      const int my_slot = my_row - s.row0;
      float4* po = space.o + piece * (D / 4) * CK_ROWS + my_slot;
      __nv_bfloat16* dst = p.o + static_cast<int64_t>(s.q0 + token) * p.o_tok + static_cast<int64_t>(s.h * p.g + my_row - token * p.g) * p.o_head;
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
        if (mine) {
          // back into order: columns 8 i + (0, 4, 1, 5, 2, 6, 3, 7)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float e[8] = {__uint_as_float(w[8 * i]), __uint_as_float(w[8 * i + 2]), __uint_as_float(w[8 * i + 4]), __uint_as_float(w[8 * i + 6]),
                                __uint_as_float(w[8 * i + 1]), __uint_as_float(w[8 * i + 3]), __uint_as_float(w[8 * i + 5]), __uint_as_float(w[8 * i + 7])};
            if (whole) {
              reinterpret_cast<uint4*>(dst)[k * 4 + i] = make_uint4(ap_pack(e[0], e[1]), ap_pack(e[2], e[3]), ap_pack(e[4], e[5]), ap_pack(e[6], e[7]));
            } else {
              po[(k * 8 + 2 * i) * CK_ROWS] = make_float4(e[0], e[1], e[2], e[3]);
              po[(k * 8 + 2 * i + 1) * CK_ROWS] = make_float4(e[4], e[5], e[6], e[7]);
            }
          }
        }
      }
      tc_fence_before();
      if (twin) {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_joined);
      }
    }
    if (failed && lane == 0) report(p.status, DEV_TIMEOUT_EPILOGUE);
  } else if (warp < 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(CK_REGS_WIDEN));
    // ------------------------------------------------------------------ widening
    const int r = tid & 127;                                    // key row of a block, and row of a tile of Q
    constexpr int W = D / 8;                                    // words of codes in a row
    const uint32_t x7 = static_cast<uint32_t>(r & 7) << 4;
    uint8_t* q_row = sQ + r * 128;
    uint8_t* kv_row = sKV + r * 128;
    uint32_t ring = 0, qn = 0, block = 0;
    // 16 bytes of a row, chunk c of it, in a tile
    auto put = [&](uint8_t* base, int c, const uint32_t (&w)[4]) {
      *reinterpret_cast<uint4*>(base + (c >> 3) * L::SUB + ((static_cast<uint32_t>(c & 7) << 4) ^ x7)) = make_uint4(w[0], w[1], w[2], w[3]);
    };
    auto widen = [&](uint8_t* base, const uint32_t (&code)[W], const uint32_t (&par)[NG]) {
      Params16 x[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) x[g] = params16(par[g]);
#pragma unroll
      for (int i = 0; i < W; ++i) {
        // a nibble in the low bits of a number from 1024 on, or four bits up in one from 64 on: that plus the code; then the code
        // times scale plus lo in one rounding
        const __half2 m1024 = half2_of(0xe400e400u), m64 = half2_of(0xd400d400u), lo2 = half2_of(x[i * 8 / G].lo2), sc2 = half2_of(x[i * 8 / G].scale2);
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t n = e ? code[i] >> 8 : code[i];
          const __half2 a = __hfma2(__hadd2(half2_of((n & 0x000f000fu) | 0x64006400u), m1024), sc2, lo2);
          const __half2 b = __hfma2(__hadd2(half2_of((n & 0x00f000f0u) | 0x54005400u), m64), sc2, lo2);
          w[2 * e] = *reinterpret_cast<const uint32_t*>(&a);
          w[2 * e + 1] = *reinterpret_cast<const uint32_t*>(&b);
        }
        put(base, i, w);
      }
    };
    auto handed = [&](uint32_t bar) {
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    Seg s;
    for (uint32_t seg = 0; !failed && walk.next(s); ++seg) {
      const int* table = p.table + s.b * p.table_stride;
      // the row of the cache that has token t, or -1
      auto row_of = [&](int t) -> int64_t {
        if (t >= s.len) return -1;
        const int page = table[t >> p.page_shift];
        if (page < 0 || page >= p.num_pages) {
          report(p.status, DEV_BAD_PAGE);
          return -1;
        }
        return ((static_cast<int64_t>(page) * p.Hk + s.h) << p.page_shift) + (t & ((1 << p.page_shift) - 1));
      };
      auto load = [&](int64_t at, const uint8_t* codes, uint32_t (&w)[W]) {
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
          uint4 x = make_uint4(0, 0, 0, 0);
          if (at >= 0) x = *reinterpret_cast<const uint4*>(codes + at * (D / 2) + i * 16);
          w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
        }
      };
      auto load_par = [&](int64_t at, const uint32_t* par, uint32_t (&w)[NG]) {
#pragma unroll
        for (int g = 0; g < NG; ++g) w[g] = at >= 0 ? par[at * NG + g] : 0u;
      };
      uint32_t kw[W], vw[W], kp[NG], vp[NG];
      int64_t at = row_of(s.j0 * 128 + r);
      load(at, p.k_codes, kw);
      load_par(at, p.k_params, kp);
      load_par(at, p.v_params, vp);
      // ---- Q
      if (!mbar_wait(bar_q_empty, (qn & 1) ^ 1)) failed = true;
      if (__any_sync(0xffffffffu, failed)) { failed = true; break; }
      ++qn;
#pragma unroll 1
      for (int t = 0; t < (s.twin() ? 1 : 2); ++t) {
        const int my = t * 128 + r, token = (s.row0 + my) / p.g;
        const __nv_bfloat16* src = p.q + static_cast<int64_t>(s.q0 + token) * p.q_tok + static_cast<int64_t>(s.h * p.g + s.row0 + my - token * p.g) * p.q_head;
        // fp16 after scaling by a power of two: the largest of a row lies in [2^14, 2^15)
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
          uint4 x = make_uint4(0, 0, 0, 0);
          if (my < s.rows) x = reinterpret_cast<const uint4*>(src)[i];
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) top = max3(top, fabsf(__uint_as_float(w[e] << 16)), fabsf(__uint_as_float(w[e] & 0xffff0000u)));
        }
        // (rows of zeros and of infinities: e = 0; the factor is applied in two halves, each of which is a normal number)
        const int ex = static_cast<int>(__float_as_uint(top) >> 23), e = top == 0.f || ex == 255 ? 0 : max(ex, 1) - 141;
        const float down = __uint_as_float(static_cast<uint32_t>(127 - e / 2) << 23), down2 = __uint_as_float(static_cast<uint32_t>(127 - (e - e / 2)) << 23);
        s_factor[(seg & 1) * CK_ROWS + my] = p.c * __uint_as_float(static_cast<uint32_t>(127 + e / 2) << 23) * __uint_as_float(static_cast<uint32_t>(127 + e - e / 2) << 23);
#pragma unroll
        for (int i = 0; i < W; ++i) {
          uint4 x = make_uint4(0, 0, 0, 0);
          if (my < s.rows) x = reinterpret_cast<const uint4*>(src)[i];
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
          uint32_t y[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {                          // elements k and k + 4
            const uint32_t a = w[k >> 1], b = w[2 + (k >> 1)];
            const float fa = __uint_as_float(k & 1 ? a & 0xffff0000u : a << 16), fb = __uint_as_float(k & 1 ? b & 0xffff0000u : b << 16);
            y[k] = pack_half(fa * down * down2, fb * down * down2);
          }
          put(q_row + t * L::TILE, i, y);
        }
      }
      handed(bar_q_full);
      // ---- K and V, block by block
      for (int j = s.j0; j < s.j1; ++j) {
        const uint32_t slot = (block + j - s.j0) % CK_FLAGS;
        load(at, p.v_codes, vw);
        uint32_t any = 0;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const bool bad = !fits_half(vp[g], p.status);
          if (bad) vp[g] = 0;
          const uint32_t mask = __ballot_sync(0xffffffffu, bad);
          if (lane == 0) s_notes[slot * 16 + g * 4 + (warp & 3)] = mask;
          any |= mask;
        }
        if (lane == 0) reinterpret_cast<uint8_t*>(s_any + slot)[warp & 3] = any != 0;
#pragma unroll
        for (int g = 0; g < NG; ++g)
          if (!fits_half(kp[g], p.status)) kp[g] = 0x7fc07fc0u;  // NaN: so are the scores of who sees it
        {
          const uint32_t st = ring % L::STAGES, use = ring / L::STAGES;
          ++ring;
          if (!mbar_wait(bar_kv_empty + 8 * st, (use & 1) ^ 1)) failed = true;
          if (__any_sync(0xffffffffu, failed)) { failed = true; break; }
          widen(kv_row + st * L::TILE, kw, kp);
          handed(bar_kv_full + 8 * st);
        }
        int64_t next = -1;
        uint32_t vp_next[NG];
        if (j + 1 < s.j1) {
          next = row_of((j + 1) * 128 + r);
          load(next, p.k_codes, kw);
          load_par(next, p.k_params, kp);
        }
        load_par(next, p.v_params, vp_next);
        {
          const uint32_t st = ring % L::STAGES, use = ring / L::STAGES;
          ++ring;
          if (!mbar_wait(bar_kv_empty + 8 * st, (use & 1) ^ 1)) failed = true;
          if (__any_sync(0xffffffffu, failed)) { failed = true; break; }
          widen(kv_row + st * L::TILE, vw, vp);
          handed(bar_kv_full + 8 * st);
        }
        at = next;
#pragma unroll
        for (int g = 0; g < NG; ++g) vp[g] = vp_next[g];
      }
      block += s.j1 - s.j0;
    }
    if (failed && lane == 0) report(p.status, DEV_TIMEOUT_PRODUCER);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(CK_REGS_MMA));
    if (warp < 14) {
      // ------------------------------------------------------------------ MMA issuers, one per tile
      const int t = warp - 12;
      const uint32_t idesc_s = make_idesc(ACC_F32, FMT_F16, FMT_F16, 128, 128);
      const uint32_t idesc_o = make_idesc(ACC_F32, FMT_F16, FMT_F16, 128, D, 0, 1);
      const uint32_t d_s = tmem_base + t * 128, d_o = tmem_base + 256 + t * 128;
      const uint32_t q0_lo = desc_lo(smem_u32(sQ), 16), k_lo = desc_lo(smem_u32(sKV), 16), v_lo = desc_lo(smem_u32(sKV), L::SUB);
      const uint32_t s_full = bar_s_full + 8 * t, p_full = bar_p_full + 16 * t, o_full = bar_o_full + 8 * t;
      uint32_t ring = 0, qn = 0, pn = 0, turn = 0;
      Seg s;
      while (walk.next(s)) {
        if (lane == 0) {
          const bool twin = s.twin();
          const int blocks = s.j1 - s.j0, n = twin ? (blocks + 1 - t) >> 1 : blocks;        // mine
          const int turns = twin ? (blocks + 1) >> 1 : blocks;   // of each tile, after the first
          const uint32_t step = twin ? 4 : 2, first = ring + (twin ? 2 * t : 0);            // K of my block i: first + step i
          const uint32_t q_lo = q0_lo + (twin ? 0u : t * (L::TILE >> 4));
          auto kv_ready = [&](uint32_t pos) { return mma_wait(bar_kv_full + 8 * (pos % L::STAGES), (pos / L::STAGES) & 1); };
          // (what only one tile uses is given back by it alone, twice over)
          auto kv_done = [&](uint32_t pos) {
            const uint32_t bar = bar_kv_empty + 8 * (pos % L::STAGES);
            if (twin) mbar_arrive(bar);
            umma_commit(bar);
          };
          auto my_turn = [&]() { return mma_wait(bar_turn + 8 * t, (turn++ & 1) ^ (t == 0)); };
          auto your_turn = [&]() { mbar_arrive(bar_turn + 8 * (t ^ 1)); };
          auto scores = [&](uint32_t pos) {
            const uint32_t kb = k_lo + (pos % L::STAGES) * (L::TILE >> 4);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              const uint32_t off = ((k >> 2) * L::SUB + (k & 3) * 32) >> 4;
              if (k == 0) mma_ss<false>(d_s, q_lo + off, kb + off, idesc_s);
              else mma_ss<true>(d_s, q_lo + off, kb + off, idesc_s);
            }
            umma_commit(s_full);
          };
          // Also a tile without blocks of its own waits for Q, so that no issuer gets more than a segment ahead.
          failed = !mma_wait(bar_q_full, qn++ & 1);
          if (!failed && n) failed = !kv_ready(first);
          if (!failed) failed = !my_turn();
          if (!failed) {
            tc_fence_after();
            if (n) scores(first);
            your_turn();
            if (n == 1) umma_commit(bar_q_empty);
            if (n == 0) mbar_arrive(bar_q_empty);
            if (n) kv_done(first);
          }
          for (int i = 0; i < n && !failed; ++i) {
            const uint32_t vpos = first + step * i + 1, kpos = first + step * (i + 1);
            if (!kv_ready(vpos) || (i + 1 < n && !kv_ready(kpos)) || !mma_wait(p_full, pn & 1) || !my_turn()) { failed = true; break; }
            tc_fence_after();
            const uint32_t vb = v_lo + (vpos % L::STAGES) * (L::TILE >> 4);
            // 16 keys per product, half of them with each part of P
#pragma unroll
            for (int k = 0; k < 4; ++k) mma_ts(d_o, d_s + k * 8, vb + k * 128, idesc_o, k || i);
            if (!mma_wait(p_full + 8, pn++ & 1)) { failed = true; break; }
            tc_fence_after();
#pragma unroll
            for (int k = 4; k < 8; ++k) mma_ts(d_o, d_s + k * 8, vb + k * 128, idesc_o, 1);
            if (i + 1 < n) scores(kpos);
            else umma_commit(o_full);
            your_turn();
            kv_done(vpos);
            if (i + 1 < n) kv_done(kpos);
            if (i + 2 == n) umma_commit(bar_q_empty);
          }
          for (int i = n; i < turns && !failed; ++i) {
            failed = !my_turn();
            your_turn();
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

// Joins the pieces of the item that begins in CTA blockIdx.x without ending there: the following CTAs' first pieces, in order.  A
// thread per row and 16 columns.
template <int D>
__global__ void __launch_bounds__(CK_ROWS) attn_chunk_join_kernel(const __grid_constant__ ChunkParams p, const int ctas) {
  wait_for_predecessor();
  const ChunkSpace<D> space(p.ws, ctas);
  const int c0 = blockIdx.x, row = threadIdx.x, col = blockIdx.y * 16;
  const Note note = space.note[c0];
  if (row >= note.rows) return;
  float m = -INFINITY, l = 0.f;
  float4 a[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) a[k] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int c = c0; c < ctas; ++c) {
    const int64_t piece = 2 * static_cast<int64_t>(c) + (c == c0);
    const float2 x = space.ml[piece * CK_ROWS + row];
    float4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = space.o[(piece * (D / 4) + col / 4 + k) * CK_ROWS + row];
    const int ends = c == c0 ? 0 : space.note[c].ends;
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
    if (ends) break;
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
  static std::atomic<int> regs{0};
  if (regs.load(std::memory_order_relaxed) == 0) {
    cudaFuncAttributes a;
    const cudaError_t e = cudaFuncGetAttributes(&a, kern);
    if (e != cudaSuccess) return e;
    regs.store(a.numRegs, std::memory_order_relaxed);
  }
  if (regs.load(std::memory_order_relaxed) < CK_REGS) return cudaErrorLaunchOutOfResources;
  cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), ChunkLayout<D>::SMEM);
  if (e != cudaSuccess) return e;
  if (!std::is_same<List, ListShared>::value) {
    e = launch_following(attn_chunk_list_kernel<D>, dim3(1), CK_THREADS, 0, s, p, ctas);
    if (e != cudaSuccess) return e;
  }
  e = launch_following(kern, dim3(static_cast<unsigned>(ctas)), CK_THREADS, ChunkLayout<D>::SMEM, s, p);
  if (e != cudaSuccess || ctas == 1) return e;
  return launch_following(attn_chunk_join_kernel<D>, dim3(static_cast<unsigned>(ctas), D / 16), CK_ROWS, 0, s, p, ctas);
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

// Items per head there can be at most (a sequence's last one may be short), and CTAs for them: one an SM, or one for every p.least
// blocks of keys where that is fewer.
int64_t attn_chunk_items(int64_t q_tokens, int B, int g) { return q_tokens * g / CK_ROWS + B; }
int attn_chunk_ctas(int64_t items, int Hk, int max_len, int least, int num_sms) {
  const int64_t units = items * Hk * ((max_len + 127) / 128 + 1), want = (units + least - 1) / least;
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
