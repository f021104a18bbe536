// Eviction from the paged 4-bit cache: per (sequence, key/value head) the newest tokens and those of the largest scores stay.
//
// Survivors in positions below the new length stay where they are; the holes between them are filled, in order, with the
// survivors from behind.  Attention does not mind the order of the keys it sees (their rotation is in them), and so a few
// rows move where closing up the ranks would move nearly all; sources and destinations are different positions, so that
// rows are moved in place by any number of threads at once.
//
//   select   a cluster per (sequence, head): the threshold by radix, eight bits a pass from the top, over keys that order like
//            the scores; the counts of a cluster's CTAs are joined through distributed shared memory.  Equal keys: the
//            lowest positions stay, by an ordered count.  Writes, for every new position, the position its token has now.
//   move     rows of codes, parameters and scores, 16 bytes a thread, on the whole GPU.
//
// Bound: the scores read once and the kept rows read and written once; what it takes is a chain of latencies (six
// barriers, of the cluster where there is one, and seven passes over the keys) and a launch.  Scores are read once, and their keys kept in shared memory while they fit.
// Measured, select and move as single launches with a cold cache: from 131071 tokens x 8 heads of 128 to 8192: 38 us and 12; 48 sequences of up to 4099 x 8 heads
// of 64 to 2048: 30 and 25; 5 sequences of up to 300 x 8 heads of 128 to 256: 14 and 8.  Called in a row 40, 47 and 14 for both together,
// and in place, scores of given-up positions zeroed and few rows moved, 45, 47 and 16 one call at a time.  Reading the counts of all CTAs at once, and other
// unrollings of the passes, changed nothing.
#include "ptx.cuh"
#include "serving.cuh"

namespace gc {

namespace {
constexpr int EV_KEYS = 40960;               // keys of a CTA that are kept in shared memory (160 KB)
constexpr int EV_MOVE_THREADS = 256;

// Larger scores have larger keys, NaN the largest; zeros are equal.
__device__ __forceinline__ uint32_t key_of(float f) {
  if (f != f) return 0xffffffffu;
  const uint32_t u = __float_as_uint(f == 0.f ? 0.f : f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint32_t ld_remote(uint32_t cluster_addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t cluster_nctarank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
// Where position t of a table's row lies (in rows of a head), or -1 for a page that is none.
__device__ __forceinline__ int64_t place(const EvictParams& p, const int* row, int h, int t) {
  const int page = row[t >> p.page_shift];
  if (page < 0 || page >= p.num_pages) {
    report(p.status, DEV_BAD_PAGE);
    return -1;
  }
  return ((static_cast<int64_t>(page) * p.Hk + h) << p.page_shift) + (t & ((1 << p.page_shift) - 1));
}
// Keys of positions t .. t + 3, t a multiple of four.
__device__ __noinline__ uint4 keys_of(const EvictParams& p, const int* row, int h, int t) {
  const int64_t at = place(p, row, h, t);
  if (at < 0) return make_uint4(0, 0, 0, 0);
  const float4 f = *reinterpret_cast<const float4*>(p.scores + at);
  return make_uint4(key_of(f.x), key_of(f.y), key_of(f.z), key_of(f.w));
}
__device__ __forceinline__ int length_of(const EvictParams& p, int b) {
  const int len = p.lengths[b];
  return len < 0 ? 0 : min(len, p.max_len);
}
}  // namespace

template <int EV_THREADS>
__global__ void __launch_bounds__(EV_THREADS) kv4_evict_select_kernel(const __grid_constant__ EvictParams p) {
  constexpr int EV_WARPS = EV_THREADS / 32;
  extern __shared__ uint4 s_keys4[];                             // [min(positions of this CTA, EV_KEYS)]
  __shared__ uint32_t s_hist[4][256];                            // one a pass: a pass ends with one cluster barrier
  __shared__ uint32_t s_warp[8];
  __shared__ int s_found[2];                                     // digit, elements still wanted below it
  __shared__ int s_equal[EV_WARPS], s_holes[EV_WARPS], s_movers[EV_WARPS];
  __shared__ uint32_t s_counts[2];                               // holes, movers of this CTA
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int ranks = static_cast<int>(cluster_nctarank()), rank = static_cast<int>(cluster_ctarank());
  const int unit = blockIdx.x / ranks, b = unit / p.Hk, h = unit - b * p.Hk;
  for (int i = tid; i < 4 * 256; i += EV_THREADS) (&s_hist[0][0])[i] = 0;
  wait_for_predecessor();
  const int n = length_of(p, b), m = min(n, p.keep);
  int* kept = p.kept + static_cast<int64_t>(unit) * p.keep;
  if (h == 0 && rank == 0 && tid == 0) {
    if (p.lengths[b] != n) report(p.status, DEV_BAD_LENGTH);
    p.out_lengths[b] = m;
  }
#pragma unroll 1
  for (int i = m + rank * EV_THREADS + tid; i < p.keep; i += ranks * EV_THREADS) kept[i] = -1;
  if (n <= p.keep) {                                             // (the same for the whole cluster)
    for (int i = rank * EV_THREADS + tid; i < n; i += ranks * EV_THREADS) kept[i] = i;
    return;
  }
  // ---- the candidates, and my stretch of them: a warp's part is a multiple of 128
  const int* row = p.table + b * p.table_stride;
  const int cand = n - p.recent;                                 // positions from here on stay
  const int share = ((cand + ranks * EV_WARPS - 1) / (ranks * EV_WARPS) + 127) & ~127;      // of a warp: four positions a lane at a time
  const int base = rank * EV_WARPS * share;                      // first of this CTA's
  const int mine = max(0, min(cand - base, EV_WARPS * share));
  const bool held = EV_WARPS * share <= p.held_keys;
  // keys of positions i .. i + 3, zeros behind `end`; and how many of the four there are
  auto keys_at = [&](int i, int end, uint32_t (&key)[4]) {
    const int there = min(max(end - i, 0), 4);
    if (held) {
      const uint4 x = there ? s_keys4[i >> 2] : make_uint4(0, 0, 0, 0);
      key[0] = x.x; key[1] = x.y; key[2] = x.z; key[3] = x.w;
    } else {
      const uint4 x = there ? keys_of(p, row, h, base + i) : make_uint4(0, 0, 0, 0);
      key[0] = x.x; key[1] = x.y; key[2] = x.z; key[3] = x.w;
    }
    return there;
  };
  if (held) {
    // the pages of several fours first, then their scores: two latencies, whatever the length
    constexpr int FLY = 4;
#pragma unroll 1
    for (int i0 = tid * 4; i0 < mine; i0 += EV_THREADS * 4 * FLY) {
      int64_t at[FLY];
      float4 f[FLY];
#pragma unroll
      for (int k = 0; k < FLY; ++k) {
        const int i = i0 + k * EV_THREADS * 4;
        const int page = i < mine ? row[(base + i) >> p.page_shift] : -1;
        at[k] = page < 0 || page >= p.num_pages ? -1 : ((static_cast<int64_t>(page) * p.Hk + h) << p.page_shift) + ((base + i) & ((1 << p.page_shift) - 1));
        if (at[k] < 0 && i < mine) report(p.status, DEV_BAD_PAGE);
      }
#pragma unroll
      for (int k = 0; k < FLY; ++k) f[k] = at[k] < 0 ? make_float4(0.f, 0.f, 0.f, 0.f) : *reinterpret_cast<const float4*>(p.scores + at[k]);
#pragma unroll
      for (int k = 0; k < FLY; ++k) {
        const int i = i0 + k * EV_THREADS * 4;
        if (i < mine) s_keys4[i >> 2] = at[k] < 0 ? make_uint4(0, 0, 0, 0) : make_uint4(key_of(f[k].x), key_of(f[k].y), key_of(f[k].z), key_of(f[k].w));
      }
    }
  }
  __syncthreads();
  // ---- the key of the last token that stays, eight bits at a time
  uint32_t prefix = 0;
  int want = p.keep - p.recent;                                  // tokens still to be found among those with this prefix
#pragma unroll 1
  for (int pass = 0; pass < 4; ++pass) {
    const int shift = 24 - 8 * pass;
    const uint32_t known = pass ? 0xffffffffu << (shift + 8) : 0u;
    uint32_t* hist = s_hist[pass];
#pragma unroll 1
    for (int i0 = warp * 128; i0 < mine; i0 += EV_THREADS * 4) {
      uint32_t key[4], digit[4];
      const int there = keys_at(i0 + lane * 4, mine, key);
      bool todo[4], some = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        todo[e] = e < there && ((key[e] ^ prefix) & known) == 0;
        digit[e] = key[e] >> shift & 255u;
        some |= todo[e];
      }
      // Scores are much alike in their leading bits: the digit of the first lane that has one is counted once for the warp, twice over.
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t rest = __ballot_sync(0xffffffffu, some);
        if (rest == 0) break;
        const int first = __ffs(rest) - 1;
        const uint32_t d = __shfl_sync(0xffffffffu, todo[0] ? digit[0] : todo[1] ? digit[1] : todo[2] ? digit[2] : digit[3], first);
        int same = 0;
        some = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool is = todo[e] && digit[e] == d;
          same += is;
          if (is) todo[e] = false;
          some |= todo[e];
        }
        same = __reduce_add_sync(0xffffffffu, same);
        if (lane == first) atomicAdd(&hist[d], static_cast<uint32_t>(same));
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (todo[e]) atomicAdd(&hist[digit[e]], 1u);
    }
    cluster_sync_all();
    // all CTAs' counts, and the digit at which the counts from the top reach what is wanted
    if (tid < 256) {
      uint32_t sum = 0;
      const uint32_t at = smem_u32(&hist[tid]);
      for (int r = 0; r < ranks; ++r) sum += ld_remote(mapa_shared(at, r));
      uint32_t incl = sum;                                       // of the digits above in this warp, and itself
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_down_sync(0xffffffffu, incl, d);
        if (lane + d < 32) incl += o;
      }
      if (lane == 0) s_warp[warp] = incl;
      asm volatile("bar.sync 1, 256;" ::: "memory");
      uint32_t above = incl - sum;
      for (int w = warp + 1; w < 8; ++w) above += s_warp[w];
      if (static_cast<int>(above) < want && want <= static_cast<int>(above + sum)) {
        s_found[0] = tid;
        s_found[1] = want - static_cast<int>(above);
      }
    }
    __syncthreads();
    if (want == 0) break;                                        // (the same for the whole cluster)
    prefix |= static_cast<uint32_t>(s_found[0]) << shift;
    want = s_found[1];
    __syncthreads();
  }
  // A key above `prefix` stays, and so do the first `want` that equal it; where none was wanted, no candidate does.
  const bool none = p.keep == p.recent;
  // ---- equal keys ahead of this warp's stretch
  const int w0 = warp * share, w1 = min(w0 + share, mine);       // of this warp, relative to `base`
  int equal_before = 0;
  if (!none) {
    int c = 0;
#pragma unroll 1
    for (int i0 = w0; i0 < w1; i0 += 128) {
      uint32_t key[4];
      const int there = keys_at(i0 + lane * 4, w1, key);
#pragma unroll
      for (int e = 0; e < 4; ++e) c += e < there && key[e] == prefix;
    }
    c = __reduce_add_sync(0xffffffffu, c);
    if (lane == 0) s_equal[warp] = c;
    const uint32_t at = smem_u32(&s_hist[3][prefix & 255u]);     // the last pass counted just the equal ones
    for (int r = lane; r < rank; r += 32) equal_before += static_cast<int>(ld_remote(mapa_shared(at, r)));
#pragma unroll
    for (int d = 16; d; d >>= 1) equal_before += __shfl_xor_sync(0xffffffffu, equal_before, d);
    __syncthreads();
    for (int w = 0; w < warp; ++w) equal_before += s_equal[w];
  }
  // Sum of v over the lanes before this one; *all: over the warp.
  auto scan = [&](int v, int* all) {
    int incl = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    *all = __shfl_sync(0xffffffffu, incl, 31);
    return incl - v;
  };
  // f(first of four positions, which of them there are, which of these stay), in order
  auto walk = [&](auto f) {
    int eq = equal_before;
#pragma unroll 1
    for (int i0 = w0; i0 < w1; i0 += 128) {
      uint32_t key[4];
      const int i = i0 + lane * 4, there = keys_at(i, w1, key);
      int same = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) same += !none && e < there && key[e] == prefix;
      int rank = 0, all = 0;
      if (__any_sync(0xffffffffu, same)) rank = scan(same, &all);
      rank += eq;
      uint32_t stays = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (none || e >= there) continue;
        if (key[e] > prefix || (key[e] == prefix && rank < want)) stays |= 1u << e;
        rank += key[e] == prefix;
      }
      eq += all;
      f(base + i, (1u << there) - 1u, stays);
    }
  };
  // of four positions from t on, those below the new length
  auto below = [&](int t) { return t + 4 <= p.keep ? 15u : t >= p.keep ? 0u : (1u << (p.keep - t)) - 1u; };
  int holes = 0, movers = 0;
  walk([&](int t, uint32_t there, uint32_t stays) {
    holes += __popc(there & ~stays & below(t));
    movers += __popc(stays & ~below(t));
  });
  holes = __reduce_add_sync(0xffffffffu, holes);
  movers = __reduce_add_sync(0xffffffffu, movers);
  if (lane == 0) {
    s_holes[warp] = holes;
    s_movers[warp] = movers;
  }
  __syncthreads();
  if (tid < 2) {
    uint32_t c = 0;
    for (int w = 0; w < EV_WARPS; ++w) c += static_cast<uint32_t>(tid == 0 ? s_holes[w] : s_movers[w]);
    s_counts[tid] = c;
  }
  cluster_sync_all();
  int hole = 0, mover = 0, all_movers = 0;                       // ahead of this warp; movers among the candidates
#pragma unroll 1
  for (int r = 0; r < ranks; ++r) {
    const int x = static_cast<int>(ld_remote(mapa_shared(smem_u32(&s_counts[0]), r))), y = static_cast<int>(ld_remote(mapa_shared(smem_u32(&s_counts[1]), r)));
    if (r < rank) {
      hole += x;
      mover += y;
    }
    all_movers += y;
  }
  for (int w = 0; w < warp; ++w) {
    hole += s_holes[w];
    mover += s_movers[w];
  }
  // ---- who stays, the holes and what moves into them
  const int lists = p.list_len;                                  // no more holes than that: kept positions, and evicted tokens
  int* hole_list = p.ws + static_cast<int64_t>(unit) * 2 * lists;
  int* mover_list = hole_list + lists;
  walk([&](int t, uint32_t there, uint32_t stays) {
    const uint32_t in = below(t), is_hole = there & ~stays & in, is_mover = stays & ~in;
    int all = 0, at = 0;                                         // holes in the lower half of a word, movers in the upper
    if (__any_sync(0xffffffffu, is_hole | is_mover)) at = scan(__popc(is_hole) | __popc(is_mover) << 16, &all);
    int hole_at = hole + (at & 0xffff), mover_at = mover + (at >> 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (stays & in & 1u << e) kept[t + e] = t + e;
      if (is_hole & 1u << e) hole_list[hole_at++] = t + e;
      if (is_mover & 1u << e) mover_list[mover_at++] = t + e;
    }
    if (p.in_place && (there & ~stays & ~in)) {                  // positions that are given up: their scores are zero from now on
      const int64_t to = place(p, row, h, t);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (to >= 0 && (there & ~stays & ~in & 1u << e)) p.scores[to + e] = 0.f;
    }
    hole += all & 0xffff;
    mover += all >> 16;
  });
#pragma unroll 1
  for (int t = cand + rank * EV_THREADS + tid; t < n; t += ranks * EV_THREADS) {
    if (t < p.keep) kept[t] = t;
    else mover_list[all_movers + t - max(cand, p.keep)] = t;
  }
  cluster_sync_all();                                            // also: no CTA leaves before the others have read its counts
  const int count = all_movers + n - max(cand, p.keep);
#pragma unroll 1
  for (int i = rank * EV_THREADS + tid; i < count; i += ranks * EV_THREADS) kept[__ldcg(hole_list + i)] = __ldcg(mover_list + i);
}

// One new position for every TPR threads: 16 bytes of codes each, keys in the lower half of them; then the parameters and the score.
// Behind the positions: the scores of what is left of the last page.
template <int D, int G>
__global__ void __launch_bounds__(EV_MOVE_THREADS) kv4_evict_move_kernel(const __grid_constant__ EvictParams p) {
  constexpr int CH = D / 32, TPR = D == 64 ? 4 : 8, NG = D / G, ITEMS = 2, ROWS = EV_MOVE_THREADS / TPR;
  wait_for_predecessor();
  const int j = threadIdx.x % TPR;
  const uint32_t rows = static_cast<uint32_t>(p.B) * p.Hk * p.keep;                 // (below 2^31)
  const uint32_t r0 = blockIdx.x * (ROWS * ITEMS) + threadIdx.x / TPR;
  int64_t from[ITEMS], to[ITEMS];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const uint32_t r = r0 + k * ROWS;
    from[k] = to[k] = -1;
    if (r >= rows) continue;
    const int unit = static_cast<int>(r / static_cast<uint32_t>(p.keep)), i = static_cast<int>(r - static_cast<uint32_t>(unit) * p.keep);
    const int b = unit / p.Hk, h = unit - b * p.Hk;
    const int t = p.kept[r];
    if (t < 0 || (p.in_place && t == i)) continue;
    from[k] = place(p, p.table + b * p.table_stride, h, t);
    to[k] = place(p, p.out_table + b * p.out_stride, h, i);
    if (to[k] < 0) from[k] = -1;
  }
  uint4 code[ITEMS];
  uint32_t par[ITEMS][NG];
  float score[ITEMS];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    if (from[k] < 0) continue;
    if (j < 2 * CH) code[k] = *reinterpret_cast<const uint4*>((j < CH ? p.k_codes : p.v_codes) + from[k] * (D / 2) + (j % CH) * 16);
    if (j < 2) {
#pragma unroll
      for (int g = 0; g < NG; ++g) par[k][g] = (j == 0 ? p.k_params : p.v_params)[from[k] * NG + g];
    }
    if (j == 2) score[k] = p.scores[from[k]];
  }
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    if (from[k] < 0) continue;
    if (j < 2 * CH) *reinterpret_cast<uint4*>((j < CH ? p.k_codes : p.v_codes) + to[k] * (D / 2) + (j % CH) * 16) = code[k];
    if (j < 2) {
#pragma unroll
      for (int g = 0; g < NG; ++g) (j == 0 ? p.k_params : p.v_params)[to[k] * NG + g] = par[k][g];
    }
    if (j == 2) {
      p.scores[to[k]] = score[k];
      if (p.in_place) p.scores[from[k]] = 0.f;                   // (no other thread reads or writes it)
    }
  }
  if (p.in_place) return;
  const int page = 1 << p.page_shift;
  for (int64_t x = static_cast<int64_t>(blockIdx.x) * EV_MOVE_THREADS + threadIdx.x; x < static_cast<int64_t>(p.B) * p.Hk << p.page_shift;
       x += static_cast<int64_t>(gridDim.x) * EV_MOVE_THREADS) {
    const int unit = static_cast<int>(x >> p.page_shift), b = unit / p.Hk, h = unit - b * p.Hk;
    const int m = min(length_of(p, b), p.keep), t = (m & ~(page - 1)) + static_cast<int>(x & (page - 1));
    if ((m & (page - 1)) == 0 || t < m) continue;
    const int64_t at = place(p, p.out_table + b * p.out_stride, h, t);
    if (at >= 0) p.scores[at] = 0.f;
  }
}

namespace {
template <int D, int G>
cudaError_t move(const EvictParams& p, cudaStream_t s) {
  constexpr int64_t PER = EV_MOVE_THREADS / (D == 64 ? 4 : 8) * 2;
  const int64_t blocks = (static_cast<int64_t>(p.B) * p.Hk * p.keep + PER - 1) / PER;
  return launch_following(kv4_evict_move_kernel<D, G>, dim3(static_cast<unsigned>(blocks)), EV_MOVE_THREADS, 0, s, p);
}
}  // namespace

// CTAs to a cluster: as many as give each SM work, where a CTA has at least 1024 positions.
// (Up to 16 of them: 69 us instead of 44 for 131071 tokens x 8 heads, with the move, for few such clusters run at once; 35 instead of 39 for one head.)
int evict_ranks(int64_t units, int max_len, int num_sms) {
  int ranks = 1;
  while (ranks < 8 && units * ranks * 2 <= 2 * num_sms && max_len >= 2048 * ranks) ranks *= 2;
  return ranks;
}

cudaError_t launch_kv4_evict(EvictParams p, int D, int G, int num_sms, cudaStream_t s) {
  const int64_t units = static_cast<int64_t>(p.B) * p.Hk;
  const int ranks = evict_ranks(units, p.max_len, num_sms);
  // 256 threads where a CTA has up to 4096 positions (four at a time and thread), and up to 16384 where more CTAs than the GPU holds
  // of the larger ones share it (40 sequences of 5000 x 8 heads: 49 us instead of 69 with the move; of 16384: 184, 187; of 40000, whose
  // keys fill an SM: 574, 335); else 1024.
  const bool few = p.max_len <= 4096 * static_cast<int64_t>(ranks) || (p.max_len <= 16384 * static_cast<int64_t>(ranks) && units * ranks > 2 * num_sms);
  const int threads = few ? 256 : 1024, warps = threads / 32;
  const int64_t need = static_cast<int64_t>((p.max_len + ranks * warps - 1) / (ranks * warps) + 127) / 128 * 128 * warps;
  p.held_keys = static_cast<int>(need < EV_KEYS ? need : EV_KEYS);
  auto kern = few ? kv4_evict_select_kernel<256> : kv4_evict_select_kernel<1024>;
  cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), EV_KEYS * 4);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(units * ranks));
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = static_cast<size_t>(p.held_keys) * 4;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(ranks);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, kern, p);
  if (e != cudaSuccess || p.keep == 0) return e;
  if (D == 64) return G == 32 ? move<64, 32>(p, s) : move<64, 64>(p, s);
  if (D == 96) return move<96, 32>(p, s);
  return G == 32 ? move<128, 32>(p, s) : G == 64 ? move<128, 64>(p, s) : move<128, 128>(p, s);
}

}  // namespace gc
