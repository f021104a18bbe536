// The attention weight every cached token receives from the queries of a step, added to what it has received before:
//
//   w[t, hk] = decay w[t, hk] + sum over queries j and the heads h that share hk of 2^(c (q[j, h] . K[t]) - lse[j, h] log2(e))
//
// lse, the logarithm of the sum of a row's exponentials, comes from the attention call before, so that tokens do not depend
// on one another: one pass over the keys, no joining.  Bound by that pass.  Scores are those of the cache attention, by the same means: the
// codes are masked out of their words as subnormal fp16 numbers and multiplied on the tensor cores with queries that are
// fp16 after scaling by a power of two, scales and offsets are applied to the sums (kernels_attn_kv4.cu has the details).
//
//   * The 32-token tiles of all (sequence, head) stand in one row, of which every warp takes an equal stretch.
//   * A lane loads its words of a tile straight into registers, a tile ahead, and calls them into the L2 four tiles ahead: with 64 elements to a group eight bytes of eight
//     rows, whole sectors.  No shared memory for keys, no barriers.
//   * The queries of up to 64 columns, as operands, stand in the warp's own shared memory; more columns than that
//     take further passes over the stretch, which add to the first one's weights.
//   * After the columns are summed, lane (gr, tg) has the sum of one token: weights are read and written 32 to a request.
//
// Measured, calls in a row: 64 sequences of up to 8192 tokens, 32 / 8 heads of 128, one query each: 90 us, 1.9 TB/s.  Neither the memory nor the
// issue of instructions (about 570 a tile, 0.38 a clock and scheduler) is at its limit: with 12 warps an SM, 18 % of what it holds, loads
// and results are waited for.  16 queries of one of 65000, 16 / 4 heads: 35 us, four or five tiles a warp behind 64 columns that every
// warp prepares for itself; 5 sequences of up to 300: 7.2 us, a launch and a chain of latencies.  Keys through a ring of asynchronous copies in shared memory: 88 us for the first, but 8.8 for the last.
#include <cuda_fp16.h>

#include "ptx.cuh"
#include "serving.cuh"

namespace gc {

namespace {
constexpr int WG_WARPS = 4, WG_THREADS = WG_WARPS * 32;
constexpr int WG_TILE = 32;
constexpr int WG_START = 3;                  // what beginning a (sequence, head) costs, in tiles
constexpr int WG_FETCH = 4;                  // tiles ahead that are called into the L2
constexpr int WG_CHUNKS = 8;                 // groups of eight columns in one pass

constexpr int WG_BLOCKS = 3;                 // CTAs an SM the registers are cut for (four of them: 101 us for the batch of 64, against 90)

template <int D, int G>
struct WeighLayout {
  static constexpr int NG = D / G, KW = D / 32;
  // operands [KW][32 lanes] of 16 bytes; then per column: NG sums, factor, offset, limit
  static constexpr int CHUNK = KW * 512 + (NG + 3) * 32;
};

__device__ __forceinline__ float wg_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void wg_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float wg_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float wg_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ int length_of(const WeighParams& p, int b) {
  const int len = p.lengths[b];
  return len < 0 ? 0 : min(len, p.max_len);
}
// Tiles of a sequence and head in the row of tiles: a few empty ones ahead of a sequence's own stand for its beginning.
__device__ __forceinline__ int tiles_of(const WeighParams& p, int b) {
  const int len = length_of(p, b);
  return len ? (len + WG_TILE - 1) / WG_TILE + WG_START : 0;
}

// A tile's keys as a lane holds them: words of rows gr, gr + 8, gr + 16, gr + 24, their parameters, and the weight of its token.
template <int D, int G>
struct Tile {
  uint32_t k[4][D / 32];
  uint32_t par[4][D / G];
  float weight;
  int64_t at;                                // where that weight lies; -1: behind the sequence
};
}  // namespace

template <int D, int G, int NT>
__global__ void __launch_bounds__(WG_THREADS, WG_BLOCKS) kv4_weigh_kernel(const __grid_constant__ WeighParams p) {
  using L = WeighLayout<D, G>;
  constexpr int NG = L::NG, KW = L::KW, KP = G >= 64 ? 2 : 1;
  extern __shared__ uint4 smem_u4[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane >> 2, tg = lane & 3;
  const int columns = p.n * p.g, held = min((columns + 8 * NT - 1) / (8 * NT) * NT, WG_CHUNKS);        // chunks in shared memory
  uint8_t* smem = reinterpret_cast<uint8_t*>(smem_u4) + warp * held * L::CHUNK;
  wait_for_predecessor();

  // ---- my stretch of the row of tiles, and the sequence it begins in
  int64_t total = 0;
#pragma unroll 1
  for (int s = lane; s < p.B; s += 32) {
    total += tiles_of(p, s);
    if (blockIdx.x == 0 && warp == 0 && p.lengths[s] != length_of(p, s)) report(p.status, DEV_BAD_LENGTH);
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
  total *= p.Hk;
  const int64_t warps = static_cast<int64_t>(gridDim.x) * WG_WARPS, me = static_cast<int64_t>(blockIdx.x) * WG_WARPS + warp;
  const int64_t each = (total >> 32) == 0 ? static_cast<int64_t>(static_cast<uint32_t>(total) / static_cast<uint32_t>(warps)) : total / warps, rest = total - each * warps;
  int64_t cur = each * me + min(me, rest);
  int64_t left = each + (me < rest);
  if (left == 0) return;
  int b = 0;
#pragma unroll 1
  for (int s0 = 0; s0 < p.B; s0 += 32) {
    const int s = s0 + lane;
    const int64_t own = s < p.B ? static_cast<int64_t>(tiles_of(p, s)) * p.Hk : 0;
    int64_t incl = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    const uint32_t hit = __ballot_sync(0xffffffffu, incl > cur);
    if (hit) {
      const int w = __ffs(hit) - 1;
      b = s0 + w;
      cur -= __shfl_sync(0xffffffffu, incl - own, w);
      break;
    }
    cur -= __shfl_sync(0xffffffffu, incl, 31);
  }
  int len = length_of(p, b), nb = tiles_of(p, b), h = static_cast<int>(static_cast<uint32_t>(cur) / static_cast<uint32_t>(nb)), k0 = static_cast<int>(cur - static_cast<int64_t>(h) * nb);

  const int page_mask = (1 << p.page_shift) - 1;
  for (;;) {
    const int kn = static_cast<int>(min(static_cast<int64_t>(nb - k0), left));
    const int i_begin = max(k0 - WG_START, 0), i_end = k0 + kn - WG_START;            // tiles of this segment
    const int* row = p.table + b * p.table_stride;
    for (int pass = 0; pass * WG_CHUNKS * 8 < columns && i_end > i_begin; ++pass) {
      const int col_begin = pass * WG_CHUNKS * 8, chunks = min(WG_CHUNKS, (columns - col_begin + 7) / 8);
      const int padded = (chunks + NT - 1) / NT * NT;
      // ---- the queries of this pass as operands: lane (gr, tg) has column gr of a chunk
      __syncwarp();
#pragma unroll 1
      for (int ch = 0; ch < padded; ++ch) {
        uint8_t* place = smem + ch * L::CHUNK;
        const int col = col_begin + ch * 8 + gr;
        const bool ok = col < columns;
        const int qi = ok ? col / p.g : 0, hh = ok ? col - qi * p.g : 0, head = h * p.g + hh;
        const __nv_bfloat16* qrow = p.q + b * p.qb + qi * p.qn + static_cast<int64_t>(head) * p.qh;
        uint4 v[KW];
        float top = 0.f;
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          v[w] = make_uint4(0, 0, 0, 0);
          if (ok) v[w] = *reinterpret_cast<const uint4*>(qrow + (w / KP) * (32 * KP) + tg * (8 * KP) + (w % KP) * 8);
          const uint32_t x[4] = {v[w].x, v[w].y, v[w].z, v[w].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(wg_lo(x[i])), fabsf(wg_hi(x[i]))));
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // q / 2^e lies in (-1, 1); the factor is applied in two halves, each of which is a normal number
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
            y[2 * i] = wg_lo(x[i]) * down * down2;
            y[2 * i + 1] = wg_hi(x[i]) * down * down2;
          }
          uint32_t f[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float up = i & 1 ? 0x1p11f : 0x1p15f;          // the odd ones meet 16 code
            const __half2 hv = __floats2half2_rn(y[i] * up, y[i + 4] * up);
            f[i] = *reinterpret_cast<const uint32_t*>(&hv);
            ss[w * 32 / G] += (__low2float(hv) + __high2float(hv)) * (0x1p-9f / up);
          }
          *reinterpret_cast<uint4*>(place + w * 512 + lane * 16) = make_uint4(f[0], f[1], f[2], f[3]);
        }
        float* sums = reinterpret_cast<float*>(place + KW * 512);
#pragma unroll
        for (int j = 0; j < NG; ++j) {
#pragma unroll
          for (int d = 1; d < 4; d <<= 1) ss[j] += __shfl_xor_sync(0xffffffffu, ss[j], d);
          if (tg == 0) sums[j * 8 + gr] = ss[j];
        }
        if (tg == 0) {
          const float lse = ok ? p.lse[(static_cast<int64_t>(b) * p.n + qi) * p.Hq + head] : -INFINITY;
          sums[NG * 8 + gr] = p.c * 0x1p9f * __uint_as_float(static_cast<uint32_t>(127 + e / 2) << 23) * __uint_as_float(static_cast<uint32_t>(127 + e - e / 2) << 23);
          sums[(NG + 1) * 8 + gr] = -lse * 1.4426950408889634f;
          // tokens the column sees; none where there is nothing to share out
          reinterpret_cast<int*>(sums)[(NG + 2) * 8 + gr] = lse == -INFINITY ? 0 : len - (p.n - 1) + qi;
        }
      }
      __syncwarp();

      // ---- the tiles
      // page numbers of 16 tiles, two per tile, one per lane; the next 16 tiles' on their way
      auto fetch = [&](int i) {
        const int t = (i + (lane >> 1)) * WG_TILE + (lane & 1) * 16;
        return i + (lane >> 1) < i_end && t < len ? row[t >> p.page_shift] : 0;
      };
      int pages = 0, pages_next = fetch(i_begin);
      auto load = [&](int i, Tile<D, G>& x) {
        if ((i - i_begin) % 16 == 0) {
          pages = pages_next;
          if (pages < 0 || pages >= p.num_pages) {
            report(p.status, DEV_BAD_PAGE);
            pages = -1;
          }
          pages_next = fetch(i + 16);
        }
        const int w = (i - i_begin) % 16, t0 = i * WG_TILE;
        // Where the halves' rows begin.  (Rows behind the sequence lie in its last page; a half behind it may have no page: the first one's
        // rows stand in.)
        auto begin_of = [&](int page, int t) { return ((static_cast<int64_t>(page) * p.Hk + h) << p.page_shift) + (t & page_mask); };
        const int page0 = __shfl_sync(0xffffffffu, pages, 2 * w), page1 = __shfl_sync(0xffffffffu, pages, 2 * w + 1);
        const int64_t at0 = begin_of(max(page0, 0), t0), at1 = t0 + 16 < len ? begin_of(max(page1, 0), t0 + 16) : at0;
        const uint8_t* src[2] = {p.k_codes + at0 * (D / 2) + gr * (D / 2) + tg * (4 * KP), p.k_codes + at1 * (D / 2) + gr * (D / 2) + tg * (4 * KP)};
        const uint32_t* ps[2] = {p.k_params + (at0 + gr) * NG, p.k_params + (at1 + gr) * NG};
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
          for (int v = 0; v < KW; v += KP) {
            const uint8_t* a = src[r >> 1] + (r & 1) * 8 * (D / 2) + v * 16;
            if constexpr (KP == 2) {
              const uint2 y = *reinterpret_cast<const uint2*>(a);
              x.k[r][v] = y.x;
              x.k[r][v + 1] = y.y;
            } else {
              x.k[r][v] = *reinterpret_cast<const uint32_t*>(a);
            }
          }
          const uint32_t* a = ps[r >> 1] + (r & 1) * 8 * NG;
          if constexpr (NG == 4) {
            const uint4 y = *reinterpret_cast<const uint4*>(a);
            x.par[r][0] = y.x; x.par[r][1] = y.y; x.par[r][2] = y.z; x.par[r][3] = y.w;
          } else if constexpr (NG == 2) {
            const uint2 y = *reinterpret_cast<const uint2*>(a);
            x.par[r][0] = y.x; x.par[r][1] = y.y;
          } else {
#pragma unroll
            for (int j = 0; j < NG; ++j) x.par[r][j] = a[j];
          }
        }
        x.at = tg >> 1 ? (page1 < 0 ? -1 : at1) : (page0 < 0 ? -1 : at0);
        // The registers hold the next tile, whose loads should find it in the L2: the tile four on is called there.  (16 rows of codes are
        // D / 16 lines, and their parameters lie in one or two.)
        {
          const int z = (i - i_begin) + WG_FETCH, t = t0 + WG_FETCH * WG_TILE + (lane & 16), which = 2 * (z % 16) + (lane >> 4);
          const int page = __shfl_sync(0xffffffffu, z / 16 == (i - i_begin) / 16 ? pages : pages_next, which);
          if (t < len && i + WG_FETCH < i_end && page >= 0 && page < p.num_pages) {
            const int64_t at = begin_of(page, t);
            const int l = lane & 15;
            if (l < D / 16) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.k_codes + at * (D / 2) + l * 128));
            else if (l == D / 16) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.k_params + at * NG));
            else if (l == D / 16 + 1) asm volatile("prefetch.global.L2 [%0];" ::"l"(pass ? p.out + at : p.weights + at));
          }
        }
        // token (tg / 2) 16 + (tg % 2) 8 + gr of the tile is this lane's
        x.weight = 0.f;
        if (t0 + (tg >> 1) * 16 + (tg & 1) * 8 + gr >= len) x.at = -1;
        if (x.at >= 0) {
          x.at += (tg & 1) * 8 + gr;
          if (pass) x.weight = p.out[x.at];
          else if (p.decay != 0.f) x.weight = p.decay * p.weights[x.at];
        }
      };
      auto work = [&](int i, const Tile<D, G>& x) {
        const int t0 = i * WG_TILE;
        const bool edge = t0 + WG_TILE > len - (p.n - 1);        // some column may not see all of it
        float sum[4] = {0.f, 0.f, 0.f, 0.f};                     // tokens gr, gr + 8, gr + 16, gr + 24
#pragma unroll 1
        for (int ch = 0; ch < padded; ch += NT) {
          const uint8_t* place = smem + ch * L::CHUNK;
          float s[NT][2][4];
#pragma unroll
          for (int j = 0; j < NG; ++j) {
            float acc[NT][2][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int mt = 0; mt < 2; ++mt) acc[nt][mt][0] = acc[nt][mt][1] = acc[nt][mt][2] = acc[nt][mt][3] = 0.f;
#pragma unroll
            for (int w = j * (G / 32); w < (j + 1) * (G / 32); ++w) {
              uint4 f[NT];
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) f[nt] = *reinterpret_cast<const uint4*>(place + nt * L::CHUNK + w * 512 + lane * 16);
#pragma unroll
              for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                  const uint32_t ka = half ? x.k[2 * mt][w] >> 8 : x.k[2 * mt][w], kb = half ? x.k[2 * mt + 1][w] >> 8 : x.k[2 * mt + 1][w];
                  const uint32_t a0 = ka & 0x000f000fu, a1 = kb & 0x000f000fu, a2 = ka & 0x00f000f0u, a3 = kb & 0x00f000f0u;
#pragma unroll
                  for (int nt = 0; nt < NT; ++nt) wg_mma(acc[nt][mt], a0, a1, a2, a3, half ? f[nt].z : f[nt].x, half ? f[nt].w : f[nt].y);
                }
              }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const float2 sq = *reinterpret_cast<const float2*>(place + nt * L::CHUNK + KW * 512 + j * 32 + tg * 8);
#pragma unroll
              for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const uint32_t par = x.par[2 * mt + (e >> 1)][j];
                  const float off = wg_lo(par) * (e & 1 ? sq.y : sq.x);
                  s[nt][mt][e] = j == 0 ? fmaf(wg_hi(par), acc[nt][mt][e], off) : fmaf(wg_hi(par), acc[nt][mt][e], s[nt][mt][e] + off);
                }
              }
            }
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const float* at = reinterpret_cast<const float*>(place + nt * L::CHUNK + KW * 512) + NG * 8 + tg * 2;
            const float2 ce = *reinterpret_cast<const float2*>(at), off = *reinterpret_cast<const float2*>(at + 8);
            const int2 lim = *reinterpret_cast<const int2*>(at + 16);
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float w = wg_ex2(fmaf(s[nt][mt][e], e & 1 ? ce.y : ce.x, e & 1 ? off.y : off.x));
                const int r = 2 * mt + (e >> 1);
                // (columns that see nothing, padding among them, have a limit of zero or less)
                const int limit = e & 1 ? lim.y : lim.x;
                if (edge ? t0 + 8 * r + gr < limit : limit > 0) sum[r] += w;
              }
            }
          }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], 1);
          sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], 2);
        }
        const float got = tg & 2 ? (tg & 1 ? sum[3] : sum[2]) : (tg & 1 ? sum[1] : sum[0]);
        if (x.at >= 0) p.out[x.at] = x.weight + got;
      };
      Tile<D, G> x;
      load(i_begin, x);
#pragma unroll 1
      for (int i = i_begin; i < i_end; ++i) {
        Tile<D, G> y;
        if (i + 1 < i_end) load(i + 1, y);
        work(i, x);
        x = y;
      }
    }
    left -= kn;
    if (left <= 0) return;
    k0 = 0;
    if (++h == p.Hk) {
      h = 0;
      do ++b;
      while (tiles_of(p, b) == 0);                               // (tiles are left, so a sequence with some follows)
      len = length_of(p, b);
      nb = tiles_of(p, b);
    }
  }
}

namespace {
template <int D, int G, int NT>
cudaError_t run(const WeighParams& p, int num_sms, cudaStream_t s) {
  auto kern = kv4_weigh_kernel<D, G, NT>;
  const int columns = p.n * p.g, chunks = (columns + 8 * NT - 1) / (8 * NT) * NT, held = chunks < WG_CHUNKS ? chunks : WG_CHUNKS;
  const size_t smem = static_cast<size_t>(WG_WARPS) * held * WeighLayout<D, G>::CHUNK;
  cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), static_cast<size_t>(WG_WARPS) * WG_CHUNKS * WeighLayout<D, G>::CHUNK);
  if (e != cudaSuccess) return e;
  // one wave of CTAs, as many as shared memory and registers let an SM have; fewer where a warp would have less than two tiles
  int resident = WG_BLOCKS;
  const int fit = static_cast<int>(227 * 1024 / (smem + 1024));
  if (fit < resident) resident = fit;
  const int64_t most = static_cast<int64_t>(p.B) * p.Hk * ((p.max_len + WG_TILE - 1) / WG_TILE + WG_START);
  const int64_t want = (most + 2 * WG_WARPS - 1) / (2 * WG_WARPS), wave = static_cast<int64_t>(num_sms) * resident;
  return launch_following(kern, dim3(static_cast<unsigned>(want < wave ? want : wave)), WG_THREADS, smem, s, p);
}
template <int D, int G>
cudaError_t by_columns(const WeighParams& p, int num_sms, cudaStream_t s) {
  return p.n * p.g <= 8 ? run<D, G, 1>(p, num_sms, s) : run<D, G, 2>(p, num_sms, s);
}
}  // namespace

cudaError_t launch_kv4_weigh(const WeighParams& p, int D, int G, int num_sms, cudaStream_t s) {
  if (D == 64) return G == 32 ? by_columns<64, 32>(p, num_sms, s) : by_columns<64, 64>(p, num_sms, s);
  if (D == 96) return by_columns<96, 32>(p, num_sms, s);
  return G == 32 ? by_columns<128, 32>(p, num_sms, s) : G == 64 ? by_columns<128, 64>(p, num_sms, s) : by_columns<128, 128>(p, num_sms, s);
}

}  // namespace gc
