// Attention of whole prompts: sequences of any length packed one behind the other, causal or not, query heads in groups
// that share a key/value head, head width 64, 96 or 128, bf16.
//
//   O = softmax(scale Q K^T) V, blockwise over 128 keys: with m a running reference, p = 2^(c s - c m), c = scale log2(e),
//   l = sum p and O = sum p V carried along; when m is raised both are multiplied by 2^(c (m_old - m_new)).
//
// Bound by the tensor cores and, as closely, by the exponentials: per 128 x 128 scores with D = 128 two products of 512 clocks
// each against 16384 exponentials, 16 a clock: 1024 clocks.  The two have to run side by side, so a CTA owns two tiles of 128
// query rows (256 neighbouring rows of one head) and alternates: while the softmax warps of one tile turn its scores into
// probabilities, the tensor core works for the other.
//   warps 0-3, 4-7   softmax of tile 0 / 1, one query row per thread: 128 scores from tensor memory into registers at once,
//                    maximum (three-input), exponentials, row sum (two sums an instruction); the bf16 probabilities go back over
//                    the scores they came from, as the A operand of the second product in tensor memory, in two parts, so that
//                    the product with the first runs while the second is made; at the end of a tile they scale and store its O
//   warp 8           TMA producer: Q tiles, and K and V blocks through one ring
//   warps 9, 10      MMA issuers of tile 0 / 1: S = Q K^T (both operands in shared memory), O += P V (P in tensor memory, V as
//                    stored, keys along the rows).  A commit covers all that its thread has issued, so that "S complete" implies "O
//                    complete"; but only products into the same accumulator, of the same shape, are promised to run in their order.
//                    Where P lies over the scores (widths 96 and 128), S of the next block is issued once the product that
//                    reads P is complete.  The tiles' batches take turns.
// Tensor memory: two score tiles of 128 columns and two outputs of D <= 128: all 512 columns at width 128.  At 64 the 64 columns beside
// each output are free, and P has them for its own.
// How it got there, for one prompt of 16384 tokens, 16 heads of 128 (1.1 TFLOP): one issuing thread for both tiles 1148 us, with
// two threads per row 1064 (its instructions were the bottleneck: products alone took 940); an issuing thread per tile with lean
// descriptors, taking turns (both tiles' products at once complete both scores together, and the tensor core idles while
// both softmaxes run: 1242) 957; probabilities in two parts 917; one thread per row, without the votes and sums two threads
// share, 865 = 1270 TFLOP/s, the tensor pipe busy 71 % of the time (products alone: 714).  All these are replays with pauses in between, and
// without the wait between a product that reads probabilities and the scores over them.  With it 920 to 965 us called in a row = 1190 to 1140 TFLOP/s, as
// the power cap has it, and 990 replayed on its own (tensor memory has no columns for P beside the scores at this width; at 64, where it has, 750).  What is left is the way round: scores
// complete, softmax, probabilities handed over, with only two tiles to alternate between.  No gain: CTA pairs (M = 256, half
// of K and V in each CTA); part of the exponentials on the FMA pipe (865 without any exponentials as well); probabilities in four
// parts (945); two score buffers of 64 keys per tile, which takes the hand-over out of the way but makes S slower (N = 64: 1001).
//   * The reference m is raised only when a score exceeds it by 2^8 (as in the cache attention): after the first block the
//     output is almost never touched, and raising it is the softmax warps' own business - no extra role, no extra hand-over.
//   * Persistent CTAs; the work list (256 query rows of a sequence, or 128 where there is little work, times heads) is made by
//     each CTA from the sequence offsets and sorted by its number of key blocks, longest first, dealt out back and forth.  The
//     first scores of the next item are issued before the last output of the current one has been stored.  Beyond 1024 entries there is
//     no list: items go by the sequences' order, and each warp finds its next one from where the last was (64 tokens, 16 / 4
//     heads of 64: 500 prompts 209 us with the list, 1000 without it 560, 4000 2000).  The sorting compares all pairs: 11 us of a
//     call with 500 entries, 45 with 1000 (prompts of one token, 38 and 82 us in all; 148 of them, which need no order, 10).
//   * Sequences of up to 128 rows leave the second tile of their items empty, so that softmax and products take turns with
//     nothing beside them: 300 prompts of 100 tokens, 32 / 8 heads of 128, 317 us where the memory alone would be 95.
//   * Rows of another sequence may follow a sequence's own in a tile.  Foreign keys are masked by selection; foreign value
//     rows are overwritten with zeros in shared memory (0 times a stored infinity would be NaN); foreign query rows are not
//     stored.
#include <atomic>

#include "attn_tc.cuh"
#include "ptx.cuh"
#include "serving.cuh"

namespace gc {

namespace {
constexpr int AP_THREADS = 384;               // three warpgroups; the last warp only hands its registers over
constexpr int AP_MAX_LIST = 1024;                // work list entries kept (and sorted) in shared memory
constexpr float AP_RAISE = 8.0f;
// Registers a thread: what the kernel has to be compiled to, and what the softmax warpgroups take and the other one gives.  Taking
// more than the block was launched with would wait for good, so a kernel compiled to fewer is not launched.  (30 bytes a thread are
// spilled all the same.)
constexpr int AP_REGS = 168, AP_REGS_SOFTMAX = 208, AP_REGS_OTHER = 88;
static_assert(2 * AP_REGS_SOFTMAX + AP_REGS_OTHER <= 3 * AP_REGS, "the warpgroups' shares exceed the launch's registers");

template <int D>
struct PromptLayout {
  static constexpr int NSUB = (D + 63) / 64;     // 64-element sub-tiles of 128-byte rows
  static constexpr int SUB = 128 * 128;
  static constexpr int TILE = NSUB * SUB;        // 128 rows of Q, K or V
  static constexpr int STAGES = D == 64 ? 8 : 4;
  static constexpr int BARS = 2 * STAGES + 16;
  static constexpr bool OVER = D > 64;           // P lies over the scores it came from (else beside O)
  static constexpr int LIST = AP_MAX_LIST * 8;
  static constexpr size_t SMEM = 1024 + static_cast<size_t>(2 + STAGES) * TILE + LIST + BARS * 8 + 64;
};

// One sequence's rows, from its offsets; offsets that decrease or leave the tensors are cut to size.
struct Seq {
  int q0, nq, k0, nk;
};
__device__ __forceinline__ Seq seq_of(const PromptParams& p, int b) {
  Seq s;
  const int tq = static_cast<int>(p.q_tokens), tk = static_cast<int>(p.k_tokens);
  s.q0 = min(max(p.cu_q[b], 0), tq);
  s.nq = max(min(p.cu_q[b + 1], tq) - s.q0, 0);
  s.k0 = min(max(p.cu_k[b], 0), tk);
  s.nk = max(min(p.cu_k[b + 1], tk) - s.k0, 0);
  return s;
}
// Keys row i of a sequence sees.
__device__ __forceinline__ int row_limit(const PromptParams& p, const Seq& s, int i) {
  return i >= s.nq ? 0 : p.causal ? max(i + 1 + s.nk - s.nq, 0) : s.nk;
}
// 128-key blocks the tile of rows [r0, r0 + 128) needs.
__device__ __forceinline__ int tile_blocks(const PromptParams& p, const Seq& s, int r0) {
  return r0 >= s.nq ? 0 : (row_limit(p, s, min(r0 + 127, s.nq - 1)) + 127) >> 7;
}

struct Item {
  Seq s;
  int row0, head;                // first of the 256 query rows, within the sequence
  int n[2];                      // key blocks of the two tiles
  bool valid;
};
}  // namespace

template <int D>
__global__ void __launch_bounds__(AP_THREADS, 1)
attn_prompt_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                   const __grid_constant__ CUtensorMap tmV, const __grid_constant__ PromptParams p, const int listed, const int most, const int log_rows) {
  using L = PromptLayout<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = smem;                                           // [2] tiles
  uint8_t* sKV = sQ + 2 * L::TILE;                              // [STAGES] tiles
  int* s_item = reinterpret_cast<int*>(sKV + L::STAGES * L::TILE);      // sequence of each entry, then its block
  int* s_tmp = s_item + AP_MAX_LIST;
  uint64_t* bars = reinterpret_cast<uint64_t*>(s_tmp + AP_MAX_LIST);
  const uint32_t b0 = smem_u32(bars);
  // [2] each: per tile; part h of the probabilities of tile t at 8 (2 t + h)
  const uint32_t bar_q_full = b0, bar_q_empty = b0 + 16, bar_s_full = b0 + 32, bar_p_full = b0 + 48, bar_o_full = b0 + 80;
  const uint32_t bar_turn = b0 + 96;                            // [2]: the tile may issue its next batch of products
  const uint32_t bar_p_read = b0 + 112;                         // [2]: the products that read the tile's probabilities are complete
  const uint32_t bar_kv_full = b0 + 128, bar_kv_empty = bar_kv_full + 8 * L::STAGES;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + L::BARS);
  int* s_total = reinterpret_cast<int*>(tmem_slot + 1);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_q_full + 8 * i, 1);
      mbar_init(bar_q_empty + 8 * i, 1);
      mbar_init(bar_s_full + 8 * i, 1);
      mbar_init(bar_o_full + 8 * i, 1);
      mbar_init(bar_turn + 8 * i, 1);
      mbar_init(bar_p_read + 8 * i, 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(bar_p_full + 8 * i, 4);
    for (int i = 0; i < L::STAGES; ++i) {
      mbar_init(bar_kv_full + 8 * i, 1);
      mbar_init(bar_kv_empty + 8 * i, 2);                       // both tiles' issuers
    }
    fence_mbar_init();
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  if (warp == 9) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // ---- the work list
  if (warp == 0) {
    int total = 0;
    for (int s0 = 0; s0 < p.B; s0 += 32) {
      const int b = s0 + lane;
      int nb = 0;
      if (b < p.B) {
        const Seq s = seq_of(p, b);
        nb = (s.nq + (1 << log_rows) - 1) >> log_rows;
        if (blockIdx.x == 0 && (p.cu_q[b] != s.q0 || p.cu_q[b + 1] != s.q0 + s.nq || p.cu_k[b] != s.k0 || p.cu_k[b + 1] != s.k0 + s.nk))
          report(p.status, DEV_BAD_OFFSETS);
      }
      int incl = nb;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
      }
      if (listed) {
        // (overlapping sequences, an error reported above, could have more blocks than the list holds: cut off)
        for (int i = 0; i < nb && total + incl - nb + i < AP_MAX_LIST; ++i) s_tmp[total + incl - nb + i] = b << 12 | i;
      }
      total = min(total + __shfl_sync(0xffffffffu, incl, 31), most);
    }
    if (lane == 0) *s_total = total;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // Not before this block has its tensor memory: a block of the next kernel that took the columns first would wait for this
  // kernel's end, and this one for the columns.
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t tmem_base = *tmem_slot;
  const int entries = *s_total;
  const int64_t items = static_cast<int64_t>(entries) * p.Hq;
  const bool sorted = listed && items > gridDim.x;              // (with one item per CTA at most there is no order to keep)
  const int* list = sorted ? s_item : s_tmp;
  if (sorted) {
    auto cost = [&](int e) {
      const Seq s = seq_of(p, e >> 12);
      const int r0 = (e & 4095) << log_rows;
      return tile_blocks(p, s, r0) + (log_rows == 8 ? tile_blocks(p, s, r0 + 128) : 0);
    };
    // costs first (packed above the entry's number so that equal ones keep their order), then each entry's rank
    int mine[(AP_MAX_LIST + AP_THREADS - 1) / AP_THREADS], key[(AP_MAX_LIST + AP_THREADS - 1) / AP_THREADS];
#pragma unroll
    for (int k = 0; k < (AP_MAX_LIST + AP_THREADS - 1) / AP_THREADS; ++k) {
      const int e = tid + k * AP_THREADS;
      mine[k] = key[k] = 0;
      if (e < entries) {
        mine[k] = s_tmp[e];
        key[k] = cost(mine[k]);
        s_item[e] = key[k];
      }
    }
    __syncthreads();
    int rank[(AP_MAX_LIST + AP_THREADS - 1) / AP_THREADS];
#pragma unroll
    for (int k = 0; k < (AP_MAX_LIST + AP_THREADS - 1) / AP_THREADS; ++k) {
      const int e = tid + k * AP_THREADS;
      rank[k] = 0;
      if (e < entries)
        for (int f = 0; f < entries; ++f) rank[k] += s_item[f] > key[k] || (s_item[f] == key[k] && f < e);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < (AP_MAX_LIST + AP_THREADS - 1) / AP_THREADS; ++k)
      if (tid + k * AP_THREADS < entries) s_item[rank[k]] = mine[k];
    __syncthreads();
  }
  // Item number r of this CTA; called by whole warps, with r rising: beyond what the list holds, the search for an entry's sequence
  // goes on where the last one of this warp ended (from the first sequence on each time, 4000 prompts of 64 tokens, 16
  // heads, took 31 ms).
  int group = 0, before = 0;                                     // sequences from `group` on, entries ahead of them
  auto item_of = [&](int r) {
    Item it;
    const int64_t g = static_cast<int64_t>(r) * gridDim.x + ((r & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
    it.valid = g < items;
    it.n[0] = it.n[1] = 0;
    it.row0 = it.head = 0;
    it.s = Seq{0, 0, 0, 0};
    if (!it.valid) return it;
    const int e = static_cast<int>(g / p.Hq);
    it.head = static_cast<int>(g - static_cast<int64_t>(e) * p.Hq);
    int b = 0, blk = 0;
    if (listed) {
      b = list[e] >> 12;
      blk = list[e] & 4095;
    } else {
      for (; group < p.B; group += 32) {
        const int nb = group + lane < p.B ? (seq_of(p, group + lane).nq + (1 << log_rows) - 1) >> log_rows : 0;
        int incl = nb;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int o = __shfl_up_sync(0xffffffffu, incl, d);
          if (lane >= d) incl += o;
        }
        const uint32_t hit = __ballot_sync(0xffffffffu, before + incl > e);
        if (hit) {
          const int w = __ffs(hit) - 1;
          b = group + w;
          const int first = before + __shfl_sync(0xffffffffu, incl - nb, w), count = __shfl_sync(0xffffffffu, nb, w);
          blk = count - 1 - (e - first);                        // the longest rows of a sequence first
          break;
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
      }
    }
    it.s = seq_of(p, b);
    it.row0 = blk << log_rows;
    it.n[0] = tile_blocks(p, it.s, it.row0);
    it.n[1] = log_rows == 8 ? tile_blocks(p, it.s, it.row0 + 128) : 0;
    return it;
  };

  bool failed = false;
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(AP_REGS_SOFTMAX));
    // ------------------------------------------------------------------ softmax and output
    const int t = warp >> 2, row = tid & 127;
    const uint32_t t_lane = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t s_addr = t_lane + t * 128, o_addr = t_lane + 256 + t * 128, p_addr = L::OVER ? s_addr : o_addr + 64;
    uint32_t ring = 0, sn = 0, on = 0;
    const float c = p.c;
    for (int r = 0; !failed; ++r) {
      const Item it = item_of(r);
      if (!it.valid) break;
      const int my_row = it.row0 + t * 128 + row;
      const int lim = row_limit(p, it.s, my_row), n = it.n[t];
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < n; ++j) {
        if (!__all_sync(0xffffffffu, mbar_wait(bar_s_full + 8 * t, sn & 1))) { failed = true; break; }
        ++sn;
        tc_fence_after();
        uint32_t v[2][64];
        tmem_ld64(s_addr, v[0]);
        tmem_ld64(s_addr + 64, v[1]);
        const int left = lim - j * 128;
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
        if (__any_sync(0xffffffffu, (mx - m) * c > AP_RAISE)) {
          const float mn = fmaxf(m, mx);
          if (score_too_large(mn * c)) report(p.status, DEV_LARGE_SCORE);
          const float f = mn == m ? 1.f : ap_ex2((m - mn) * c);  // 0 from the initial minus infinity
          m = mn;
          l *= f;
          if (j > 0) {
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
        const float off = m == -INFINITY ? 0.f : -m * c;
        const uint64_t c2 = pair2(c, c), off2 = pair2(off, off);
        if (j * 128 + 128 > it.s.nk) {
          // the sequence ends inside this block: whatever follows it in V becomes zero
          const uint32_t pos = ring + 2 * j + 1, st = pos % L::STAGES;
          if (!__all_sync(0xffffffffu, mbar_wait(bar_kv_full + 8 * st, (pos / L::STAGES) & 1))) { failed = true; break; }
          if (j * 128 + row >= it.s.nk) {
#pragma unroll
            for (int k = 0; k < L::NSUB; ++k) {
              uint4* z = reinterpret_cast<uint4*>(sKV + st * L::TILE + k * L::SUB + row * 128);
#pragma unroll
              for (int i = 0; i < 8; ++i) z[i] = make_uint4(0, 0, 0, 0);
            }
          }
          fence_proxy_async_smem();
        }
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
            w[i] = ap_pack(e0, e1);
          }
          tmem_st32(p_addr + h * 32, w);
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
      ring += 2 * max(it.n[0], it.n[1]);
      const bool store = my_row < it.s.nq && t * 128 < 1 << log_rows;
      __nv_bfloat16* dst = p.o + static_cast<int64_t>(it.s.q0 + my_row) * p.o_tok + static_cast<int64_t>(it.head) * p.o_head;
      if (n == 0) {
        if (store) {
#pragma unroll
          for (int i = 0; i < D / 8; ++i) reinterpret_cast<uint4*>(dst)[i] = make_uint4(0, 0, 0, 0);
        }
        continue;
      }
      if (!__all_sync(0xffffffffu, mbar_wait(bar_o_full + 8 * t, on & 1))) { failed = true; break; }
      ++on;
      tc_fence_after();
      const float rl = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll 1
      for (int k = 0; k < D / 32; ++k) {
        uint32_t w[32];
        tmem_ld32(o_addr + k * 32, w);
        tmem_wait_ld();
        if (store) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = ap_pack(__uint_as_float(w[8 * i + 2 * e]) * rl, __uint_as_float(w[8 * i + 2 * e + 1]) * rl);
            reinterpret_cast<uint4*>(dst)[k * 4 + i] = make_uint4(x[0], x[1], x[2], x[3]);
          }
        }
      }
      tc_fence_before();
    }
    if (failed && lane == 0) report(p.status, DEV_TIMEOUT_EPILOGUE);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(AP_REGS_OTHER));
    if (warp == 8) {
      // ------------------------------------------------------------------ TMA producer
      uint32_t ring = 0, qn[2] = {0, 0};
      const int g = p.Hq / p.Hk;
      for (int r = 0;; ++r) {
        const Item it = item_of(r);
        if (!it.valid) break;
        if (lane == 0) {
          const int kvh = it.head / g;
          auto load_q = [&](int t) -> bool {
            if (it.n[t] == 0) return true;
            if (!mbar_wait(bar_q_empty + 8 * t, (qn[t] & 1) ^ 1)) return false;
            ++qn[t];
            mbar_arrive_expect_tx(bar_q_full + 8 * t, static_cast<uint32_t>(L::TILE));
            for (int j = 0; j < L::NSUB; ++j)
              tma_load_3d(smem_u32(sQ) + t * L::TILE + j * L::SUB, &tmQ, j * 64, it.head, it.s.q0 + it.row0 + t * 128, bar_q_full + 8 * t);
            return true;
          };
          auto load_kv = [&](const CUtensorMap* tm, int tile) -> bool {
            const uint32_t st = ring % L::STAGES, use = ring / L::STAGES;
            ++ring;
            if (!mbar_wait(bar_kv_empty + 8 * st, (use & 1) ^ 1)) return false;
            mbar_arrive_expect_tx(bar_kv_full + 8 * st, static_cast<uint32_t>(L::TILE));
            for (int j = 0; j < L::NSUB; ++j)
              tma_load_3d(smem_u32(sKV) + st * L::TILE + j * L::SUB, tm, j * 64, kvh, it.s.k0 + tile * 128, bar_kv_full + 8 * st);
            return true;
          };
          const int n = max(it.n[0], it.n[1]);
          failed = !load_q(0);
          for (int j = 0; j < n && !failed; ++j) {
            failed = !load_kv(&tmK, j);
            if (j == 0 && !failed) failed = !load_q(1);
            if (!failed) failed = !load_kv(&tmV, j);
          }
          if (failed) report(p.status, DEV_TIMEOUT_PRODUCER);
        }
        if (__any_sync(0xffffffffu, failed)) break;
      }
    } else if (warp < 11) {
      // ------------------------------------------------------------------ MMA issuers, one per tile
      const int t = warp - 9;
      const uint32_t idesc_s = make_idesc(ACC_F32, FMT_BF16, FMT_BF16, 128, 128);
      const uint32_t idesc_o = make_idesc(ACC_F32, FMT_BF16, FMT_BF16, 128, D, 0, 1);
      const uint32_t d_s = tmem_base + t * 128, d_o = tmem_base + 256 + t * 128, d_p = L::OVER ? d_s : d_o + 64;
      const uint32_t q_lo = desc_lo(smem_u32(sQ) + t * L::TILE, 16), k_lo = desc_lo(smem_u32(sKV), 16), v_lo = desc_lo(smem_u32(sKV), L::SUB);
      const uint32_t q_full = bar_q_full + 8 * t, q_empty = bar_q_empty + 8 * t, s_full = bar_s_full + 8 * t, p_full = bar_p_full + 16 * t,
                     o_full = bar_o_full + 8 * t, p_read = bar_p_read + 8 * t;
      uint32_t ring = 0, qn = 0, pn = 0, rn = 0;
      auto kv_ready = [&](uint32_t pos) { return mma_wait(bar_kv_full + 8 * (pos % L::STAGES), (pos / L::STAGES) & 1); };
      auto kv_done = [&](uint32_t pos) { umma_commit(bar_kv_empty + 8 * (pos % L::STAGES)); };
      // The tiles take turns, one batch of products (O += P V, next S) each.
      uint32_t turn = 0;
      auto my_turn = [&]() { return mma_wait(bar_turn + 8 * t, (turn++ & 1) ^ (t == 0)); };
      auto your_turn = [&]() { mbar_arrive(bar_turn + 8 * (t ^ 1)); };
      // Scores that will overwrite probabilities wait for the products that read them, the last ones this thread has committed to p_read.
      auto p_is_read = [&]() { return !L::OVER || rn == 0 || mma_wait(p_read, (rn - 1) & 1); };
      // S = Q K^T with the K block of ring position `pos`
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
      // the first scores of an item, whose first K block stands at ring position `ring`
      auto begin = [&](const Item& it) -> bool {
        const int n = t ? it.n[1] : it.n[0];
        if (n && !mma_wait(q_full, qn++ & 1)) return false;
        if (max(it.n[0], it.n[1])) {
          if (!kv_ready(ring) || (n && !p_is_read()) || !my_turn()) return false;
          tc_fence_after();
          if (n) scores(ring);
          your_turn();
          if (n == 1) umma_commit(q_empty);
          kv_done(ring);
        }
        return true;
      };
      Item it = item_of(0);
      if (it.valid && lane == 0) failed = !begin(it);
      for (int r = 0; it.valid; ++r) {
        if (__any_sync(0xffffffffu, failed)) break;
        const Item next = item_of(r + 1);
        if (lane == 0) {
          const int n = t ? it.n[1] : it.n[0], most = max(it.n[0], it.n[1]);
          // ring position of K_j: ring + 2 j, of V_j: ring + 2 j + 1
          for (int j = 0; j < most; ++j) {
            const uint32_t vpos = ring + 2 * j + 1;
            // (Also an issuer that skips a block waits until it is there: else it could get a round of the ring ahead, and its
            // next arrival would stand in for the other issuer's.)
            if (!kv_ready(vpos) || (j + 1 < most && !kv_ready(vpos + 1))) { failed = true; break; }
            if (j < n && !mma_wait(p_full, pn & 1)) { failed = true; break; }
            if (!my_turn()) { failed = true; break; }
            tc_fence_after();
            if (j < n) {
              const uint32_t vb = v_lo + (vpos % L::STAGES) * (L::TILE >> 4);
              // 16 keys per product, half of them with each part of P
#pragma unroll
              for (int k = 0; k < 4; ++k) mma_ts(d_o, d_p + k * 8, vb + k * 128, idesc_o, k || j);
              if (!mma_wait(p_full + 8, pn++ & 1)) { failed = true; break; }
              tc_fence_after();
#pragma unroll
              for (int k = 4; k < 8; ++k) mma_ts(d_o, d_p + k * 8, vb + k * 128, idesc_o, 1);
              if constexpr (L::OVER) {
                umma_commit(p_read);
                ++rn;
              }
              if (j + 1 == n) umma_commit(o_full);
              else {
                if (!p_is_read()) { failed = true; break; }
                tc_fence_after();
                scores(vpos + 1);
              }
            }
            your_turn();
            kv_done(vpos);
            if (j + 1 < most) kv_done(vpos + 1);
            if (j + 2 == n) umma_commit(q_empty);
          }
          ring += 2 * most;
          if (!failed && next.valid) failed = !begin(next);
          if (failed) report(p.status, DEV_TIMEOUT_MMA);
        }
        it = next;
      }
    }
  }
  if (failed) {                                                  // copies and products in flight come to rest before the block exits
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) {
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

template <int D>
static cudaError_t prompt_run(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const PromptParams& p, int num_sms,
                              cudaStream_t s) {
  auto kern = attn_prompt_kernel<D>;
  static std::atomic<int> regs{0};
  if (regs.load(std::memory_order_relaxed) == 0) {
    cudaFuncAttributes a;
    const cudaError_t e = cudaFuncGetAttributes(&a, kern);
    if (e != cudaSuccess) return e;
    regs.store(a.numRegs, std::memory_order_relaxed);
  }
  if (regs.load(std::memory_order_relaxed) < AP_REGS) return cudaErrorLaunchOutOfResources;
  cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), PromptLayout<D>::SMEM);
  if (e != cudaSuccess) return e;
  // 256 rows to an item, or 128 where even those leave SMs without work: the one tile then has the tensor core to itself (one
  // prompt of 1693 tokens, 2 heads of 128: 36.7, so 32.8 us; 2048, 8 heads: 36.2, so 32.9; 512, 16 heads: 15.4, so 13.4)
  // (entries: what the offsets can come to at most, for every sequence may end inside a block)
  const int log_rows = (p.q_tokens / 128 + p.B) * p.Hq <= num_sms ? 7 : 8;
  const int64_t entries = (p.q_tokens >> log_rows) + p.B;
  const int64_t items = entries * p.Hq;
  const int grid = static_cast<int>(items < num_sms ? items : num_sms);
  // the list packs a block number into 12 bits
  const int listed = entries <= AP_MAX_LIST && p.q_tokens <= 256 * 4096LL;
  return launch_following(kern, dim3(static_cast<unsigned>(grid)), AP_THREADS, PromptLayout<D>::SMEM, s, tmQ, tmK, tmV, p, listed, static_cast<int>(entries), log_rows);
}

cudaError_t launch_attn_prompt(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const PromptParams& p, int num_sms,
                               cudaStream_t s) {
  if (p.D == 64) return prompt_run<64>(tmQ, tmK, tmV, p, num_sms, s);
  if (p.D == 96) return prompt_run<96>(tmQ, tmK, tmV, p, num_sms, s);
  return prompt_run<128>(tmQ, tmK, tmV, p, num_sms, s);
}

}  // namespace gc
