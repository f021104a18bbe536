// Attention of a few new queries per sequence over the paged 4-bit cache.
//
//   o[col] = sum_t p(t, col) V[t] / sum_t p(t, col),   p = 2^(c (q[col] . K[t]) - m[col]),   K, V = lo + code * scale
//
// A column is one (query, query head) of those that share a key/value head.  The floor is the cache read once; a key
// element is half a byte, so the work per byte is what has to be kept small: at the copy bandwidth of the whole GPU an SM
// has 2.8 lane-instructions per element of K or V.
//
//   * The codes go into the matrix instruction as they are.  A nibble moved to bits 3..6 of a bf16 with exponent of 16 is
//     the number 16 + code, exactly, and one shift and one logic instruction make two of them.  Scales and offsets are
//     applied to sums, never to elements:
//       q . K[t]            = scale_t * (sum_i q_i (16 + code_i) - 16 sum_i q_i) + lo_t * sum_i q_i       per group
//       sum_t p_t V[t][d]   = sum_t p'_t (16 + code_td) + sum_t (p_t (lo_t + 7.5 scale_t) - 23.5 p'_t),   p'_t = bf16(p_t scale_t)
//     The first sum of each line is the MMA's (fp32 accumulators, -16 sum q as their initial value in the first); the
//     others are a few fp32 operations per (token, column).  p' is the only rounding before the output's; what it rounds is the
//     distance from the middle of the group's range (code - 7.5), half of what the distance from lo would lose.
//   * m16n8k16 MMAs with the codes as the 16-row operand: tokens are the rows of the first product and the reduction of the
//     second, so a lane's nibbles are always neighbours in memory (head-dimension neighbours; the order inside a reduction
//     axis is free, Q and P are permuted to match), and 8 columns cost 8, not 16.
//   * A warp is on its own: it takes every fourth 32-token tile of its CTA's range, copies tiles ahead into its own ring in
//     shared memory with 16-byte asynchronous copies, and keeps running maximum, sum and output of its columns in
//     registers.  No barrier until the end, where the warps of a CTA are joined in shared memory and the CTAs of a unit
//     (when a sequence is split) by a second small kernel in a fixed order.
//   * The running maximum is a reference that is only raised when a score exceeds it by 2^8: one vote per tile instead
//     of a reduction, and the sums stay far inside fp32.
#include "ptx.cuh"
#include "serving.cuh"

namespace gc {

namespace {
constexpr int AK_WARPS = 4;
constexpr int AK_THREADS = AK_WARPS * 32;
constexpr int AK_TILE = 32;                  // tokens per tile of a warp
constexpr int AK_STAGES = 4;
constexpr float AK_RAISE = 8.0f;             // binades a score may exceed the reference by

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
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
// nibble i of each 16-bit half as the bf16 number 16 + nibble
template <int I>
__device__ __forceinline__ uint32_t nib(uint32_t w) {
  const uint32_t s = I == 0 ? w << 3 : w >> (I == 0 ? 0 : 4 * I - 3);
  return (s & 0x00780078u) | 0x41804180u;
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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

// Byte offset of 16-byte chunk c of token row r in a codes tile.  The exclusive-or spreads the rows that one load
// instruction touches over all banks: eight rows with the same chunk (keys), rows 0..3, 4..7, ... with two neighbouring
// chunks (values).
template <int D>
__device__ __forceinline__ uint32_t code_off(int r, int c) {
  if constexpr (D == 64) return r * 32 + ((c ^ ((r >> 2) & 1)) << 4);
  const int k = (r >> 1) & 3;
  return r * 64 + ((c ^ ((k >> 1) | ((k & 1) << 1))) << 4);
}
}  // namespace

// NT: groups of eight columns per CTA
template <int D, int G, int NT>
__global__ void __launch_bounds__(AK_THREADS) attn_kv4_kernel(const __grid_constant__ Kv4AttnParams p) {
  using L = KvLayout<D, G>;
  constexpr int NG = L::NG, KW = D / 32, MT = D / 16, COLS = 8 * NT;
  constexpr int UG = G / 32;                                     // 16-bit units of V per lane, token and group
  extern __shared__ uint4 smem_u4[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(smem_u4);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane >> 2, tg = lane & 3;
  const int split = blockIdx.x % p.n_split;
  const int unit = blockIdx.x / p.n_split;                       // ((b * Hk) + hk) * col_chunks + chunk
  const int chunk = unit % p.col_chunks, bh = unit / p.col_chunks, b = bh / p.Hk, hk = bh - b * p.Hk;
  const int columns = p.n * p.g, col0 = chunk * COLS;

  int len = p.lengths[b];
  if (len < 0 || len > p.max_len) {
    if (threadIdx.x == 0) report(p.status, DEV_BAD_LENGTH);
    len = len < 0 ? 0 : p.max_len;
  }
  const int t_begin = split * p.split_len;
  const int t_end = min(len, t_begin + p.split_len);
  if (split > 0 && t_begin >= len) return;                       // the joining kernel knows which splits exist

  // Queries as the second operand of the first product: lane (gr, tg) holds of column gr the eight elements 8 tg .. 8 tg + 7
  // of every 32, in pairs (0,4), (1,5), (2,6), (3,7), the order in which the nibbles of a word come apart.
  uint32_t qf[NT][KW][4];
  float sq[NT][NG][2];                                           // sum of q over a group, columns 2 tg and 2 tg + 1
  int lim[NT][2];                                                // tokens that column sees
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int col = col0 + nt * 8 + gr;
    float s[NG];
#pragma unroll
    for (int j = 0; j < NG; ++j) s[j] = 0.f;
    const bool ok = col < columns;
    const int qi = ok ? col / p.g : 0, hh = ok ? col - qi * p.g : 0;
    const __nv_bfloat16* qrow = p.q + b * p.qb + qi * p.qn + static_cast<int64_t>(hk * p.g + hh) * p.qh;
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (ok) v = *reinterpret_cast<const uint4*>(qrow + 32 * w + 8 * tg);
      qf[nt][w][0] = __byte_perm(v.x, v.z, 0x5410);              // elements 0, 4
      qf[nt][w][1] = __byte_perm(v.x, v.z, 0x7632);              // 1, 5
      qf[nt][w][2] = __byte_perm(v.y, v.w, 0x5410);              // 2, 6
      qf[nt][w][3] = __byte_perm(v.y, v.w, 0x7632);              // 3, 7
#pragma unroll
      for (int i = 0; i < 4; ++i) s[w * 32 / G] += bf_lo(qf[nt][w][i]) + bf_hi(qf[nt][w][i]);
    }
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      s[j] += __shfl_xor_sync(0xffffffffu, s[j], 1);
      s[j] += __shfl_xor_sync(0xffffffffu, s[j], 2);
      sq[nt][j][0] = __shfl_sync(0xffffffffu, s[j], 8 * tg);
      sq[nt][j][1] = __shfl_sync(0xffffffffu, s[j], 8 * tg + 4);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int cc = col0 + nt * 8 + 2 * tg + i;
      lim[nt][i] = cc < columns ? len - (p.n - 1) + cc / p.g : 0;
    }
  }

  float o[NT][MT][4], m[NT][2], l[NT][2], z[NT][NG][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int i = 0; i < MT; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      m[nt][i] = -INFINITY;
      l[nt][i] = 0.f;
#pragma unroll
      for (int j = 0; j < NG; ++j) z[nt][j][i] = 0.f;
    }
  }

  const int tiles = t_end > t_begin ? (t_end - t_begin + AK_TILE - 1) / AK_TILE : 0;
  const int mine = tiles > warp ? (tiles - warp + AK_WARPS - 1) / AK_WARPS : 0;      // tiles warp, warp + 4, ...
  uint8_t* ring = smem + warp * L::RING;
  const uint32_t ring_a = smem_u32(ring);
  const int* trow = p.table + b * p.table_stride;
  const int page_mask = (1 << p.page_shift) - 1;

  // Page numbers of 16 tiles at a time, two per tile (a tile of 32 tokens is two pages of 16 at worst), one per lane.
  int pages = 0;
  auto fetch_pages = [&](int i) {
    const int tok = t_begin + (warp + AK_WARPS * (i + (lane >> 1))) * AK_TILE + (lane & 1) * 16;
    pages = 0;
    if (tok < t_end) {
      pages = __ldg(trow + (tok >> p.page_shift));
      if (pages < 0 || pages >= p.num_pages) {
        report(p.status, DEV_BAD_PAGE);
        pages = 0;
      }
    }
  };
  auto issue = [&](int i) {
    if (i < mine) {
      if ((i & 15) == 0) fetch_pages(i);
      const int t0 = t_begin + (warp + AK_WARPS * i) * AK_TILE;
      const uint32_t st = ring_a + (i % AK_STAGES) * L::STAGE;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int page = __shfl_sync(0xffffffffu, pages, 2 * (i & 15) + half);
        const int tok = t0 + half * 16;
        if (tok < t_end) {
          const int64_t row = ((static_cast<int64_t>(page) * p.Hk + hk) << p.page_shift) + (tok & page_mask);
          constexpr int CH = L::ROW / 16, N = 16 * CH;           // 16-byte chunks per token, per half tile
          const uint8_t* ks = p.k_codes + row * L::ROW;
          const uint8_t* vs = p.v_codes + row * L::ROW;
#pragma unroll
          for (int x0 = 0; x0 < N; x0 += 32) {
            const int x = x0 + lane;
            if (N % 32 == 0 || x < N) {
              const int r = x / CH, c = x - r * CH;
              const uint32_t off = code_off<D>(half * 16 + r, c);
              cp_async16(st + off, ks + x * 16);
              cp_async16(st + L::CODES + off, vs + x * 16);
            }
          }
          constexpr int PN = 16 * NG * 4 / 16;                   // chunks of parameters: 4 to 16
          if (lane < PN) cp_async16(st + 2 * L::CODES + half * (16 * NG * 4) + lane * 16, reinterpret_cast<const uint8_t*>(p.k_params + row * NG) + lane * 16);
          else if (lane >= 16 && lane - 16 < PN)
            cp_async16(st + 2 * L::CODES + L::PARAMS + half * (16 * NG * 4) + (lane - 16) * 16, reinterpret_cast<const uint8_t*>(p.v_params + row * NG) + (lane - 16) * 16);
        }
      }
    }
    cp_commit();
  };

#pragma unroll
  for (int i = 0; i < AK_STAGES - 1; ++i) issue(i);

  for (int i = 0; i < mine; ++i) {
    cp_wait<AK_STAGES - 2>();
    __syncwarp();
    const int t0 = t_begin + (warp + AK_WARPS * i) * AK_TILE;
    const uint32_t kc = ring_a + (i % AK_STAGES) * L::STAGE, vc = kc + L::CODES, kp = vc + L::CODES, vp = kp + L::PARAMS;

    // ---- scores of 32 tokens.  Row r of a 16-row operand is token perm(r) = r / 2 (r even), 4 + r / 2 (r odd), + 8 above
    const int pr = (gr >> 1) + ((gr & 1) << 2);
    float s[2][NT][4];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      const int ta = mt * 16 + pr;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[mt][nt][0] = s[mt][nt][1] = s[mt][nt][2] = s[mt][nt][3] = 0.f;
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        float acc[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          acc[nt][0] = acc[nt][2] = -16.f * sq[nt][j][0];
          acc[nt][1] = acc[nt][3] = -16.f * sq[nt][j][1];
        }
#pragma unroll
        for (int w = j * (G / 32); w < (j + 1) * (G / 32); ++w) {
          const uint32_t ka = lds32(kc + code_off<D>(ta, w) + tg * 4), kb = lds32(kc + code_off<D>(ta + 8, w) + tg * 4);
          const uint32_t a0 = nib<0>(ka), a1 = nib<0>(kb), a2 = nib<1>(ka), a3 = nib<1>(kb);
          const uint32_t c0 = nib<2>(ka), c1 = nib<2>(kb), c2 = nib<3>(ka), c3 = nib<3>(kb);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            mma_bf16(acc[nt], a0, a1, a2, a3, qf[nt][w][0], qf[nt][w][1]);
            mma_bf16(acc[nt], c0, c1, c2, c3, qf[nt][w][2], qf[nt][w][3]);
          }
        }
        const uint32_t pa = lds32(kp + (ta * NG + j) * 4), pb = lds32(kp + ((ta + 8) * NG + j) * 4);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          s[mt][nt][0] = fmaf(bf_hi(pa), acc[nt][0], fmaf(bf_lo(pa), sq[nt][j][0], s[mt][nt][0]));
          s[mt][nt][1] = fmaf(bf_hi(pa), acc[nt][1], fmaf(bf_lo(pa), sq[nt][j][1], s[mt][nt][1]));
          s[mt][nt][2] = fmaf(bf_hi(pb), acc[nt][2], fmaf(bf_lo(pb), sq[nt][j][0], s[mt][nt][2]));
          s[mt][nt][3] = fmaf(bf_hi(pb), acc[nt][3], fmaf(bf_lo(pb), sq[nt][j][1], s[mt][nt][3]));
        }
      }
    }
    // Some column may not see all of this tile: the columns' limits lie within n of the sequence's end, padding columns
    // see nothing and are left as they come (nobody reads them).
    const bool edge = t0 + AK_TILE > len - (p.n - 1) || t0 + AK_TILE > t_end;
    if (edge) {
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
      for (int e = 0; e < 2; ++e) {
        const float mx = fmaxf(fmaxf(s[0][nt][e], s[0][nt][e + 2]), fmaxf(s[1][nt][e], s[1][nt][e + 2]));
        over |= mx * p.c > m[nt][e] + AK_RAISE;
      }
    }
    if (__any_sync(0xffffffffu, over)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float mx = fmaxf(fmaxf(s[0][nt][e], s[0][nt][e + 2]), fmaxf(s[1][nt][e], s[1][nt][e + 2])) * p.c;
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
          const float mn = fmaxf(m[nt][e], mx);
          const float f = m[nt][e] == mn ? 1.f : ak_ex2(m[nt][e] - mn);      // 0 from the initial minus infinity
          m[nt][e] = mn;
          l[nt][e] *= f;
#pragma unroll
          for (int j = 0; j < NG; ++j) z[nt][j][e] *= f;
#pragma unroll
          for (int k = 0; k < MT; ++k) {
            o[nt][k][e] *= f;
            o[nt][k][e + 2] *= f;
          }
        }
      }
    }
    // ---- probabilities and the second product, 16 tokens at a time
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      const int ta = mt * 16 + pr;
      float pw[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float r0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0], r1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1];
        pw[nt][0] = ak_ex2(fmaf(s[mt][nt][0], p.c, -r0));
        pw[nt][1] = ak_ex2(fmaf(s[mt][nt][1], p.c, -r1));
        pw[nt][2] = ak_ex2(fmaf(s[mt][nt][2], p.c, -r0));
        pw[nt][3] = ak_ex2(fmaf(s[mt][nt][3], p.c, -r1));
        l[nt][0] += pw[nt][0] + pw[nt][2];
        l[nt][1] += pw[nt][1] + pw[nt][3];
      }
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        const uint32_t pa = lds32(vp + (ta * NG + j) * 4), pb = lds32(vp + ((ta + 8) * NG + j) * 4);
        const float ma = fmaf(7.5f, bf_hi(pa), bf_lo(pa)), mb = fmaf(7.5f, bf_hi(pb), bf_lo(pb));     // the middle of a group's range
        uint32_t bf[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float x0 = pw[nt][0] * bf_hi(pa), x1 = pw[nt][1] * bf_hi(pa), x2 = pw[nt][2] * bf_hi(pb), x3 = pw[nt][3] * bf_hi(pb);
          float y0 = pw[nt][0] * ma, y1 = pw[nt][1] * ma, y2 = pw[nt][2] * mb, y3 = pw[nt][3] * mb;
          if (edge) {                                            // a weight of zero hides whatever the cache holds there
            if (s[mt][nt][0] == -INFINITY) x0 = y0 = 0.f;
            if (s[mt][nt][1] == -INFINITY) x1 = y1 = 0.f;
            if (s[mt][nt][2] == -INFINITY) x2 = y2 = 0.f;
            if (s[mt][nt][3] == -INFINITY) x3 = y3 = 0.f;
          }
          const uint32_t ua = pack_bf16(x0, x1), ub = pack_bf16(x2, x3);
          z[nt][j][0] += fmaf(-23.5f, bf_lo(ua) + bf_lo(ub), y0 + y2);
          z[nt][j][1] += fmaf(-23.5f, bf_hi(ua) + bf_hi(ub), y1 + y3);
          bf[nt][0] = transpose8x8(ua);
          bf[nt][1] = transpose8x8(ub);
        }
        // lane (gr, tg): tokens tg, tg + 4, tg + 8, tg + 12 of the 16; elements j G + gr G / 8 + 4 u + nibble
        const int tv = mt * 16 + tg;
        uint32_t vw[4][(UG + 1) / 2];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int byte = j * (G / 2) + gr * (G / 16);
          const uint32_t a = vc + code_off<D>(tv + 4 * k, byte >> 4) + (byte & 15);
          if constexpr (UG == 1) vw[k][0] = lds16(a);
          if constexpr (UG == 2) vw[k][0] = lds32(a);
          if constexpr (UG == 4) {
            const uint2 t = lds64(a);
            vw[k][0] = t.x;
            vw[k][1] = t.y;
          }
        }
#pragma unroll
        for (int u = 0; u < UG; ++u) {
          const uint32_t sel = (u & 1) ? 0x7632u : 0x5410u;
          const uint32_t x = __byte_perm(vw[0][u >> 1], vw[1][u >> 1], sel), y = __byte_perm(vw[2][u >> 1], vw[3][u >> 1], sel);
          const uint32_t a0 = nib<0>(x), a1 = nib<1>(x), a2 = nib<0>(y), a3 = nib<1>(y);
          const uint32_t c0 = nib<2>(x), c1 = nib<3>(x), c2 = nib<2>(y), c3 = nib<3>(y);
          const int k = (j * UG + u) * 2;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            mma_bf16(o[nt][k], a0, a1, a2, a3, bf[nt][0], bf[nt][1]);
            mma_bf16(o[nt][k + 1], c0, c1, c2, c3, bf[nt][0], bf[nt][1]);
          }
        }
      }
    }
    __syncwarp();
    issue(i + AK_STAGES - 1);
  }
  cp_wait<0>();

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
          *reinterpret_cast<float4*>(row + j * G + gr * (G / 8) + 4 * u) =
              make_float4(o[nt][k][e] + z[nt][j][e], o[nt][k][e + 2] + z[nt][j][e], o[nt][k + 1][e] + z[nt][j][e], o[nt][k + 1][e + 2] + z[nt][j][e]);
        }
      }
      if (gr == 0) {
        s_m[warp * COLS + col] = m[nt][e];
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
    float ll = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < AK_WARPS; ++w) {
      const float mw = s_m[w * COLS + col];
      if (mw == -INFINITY) continue;
      const float f = ak_ex2(mw - mm);
      const float4 v = *reinterpret_cast<const float4*>(s_o + (w * COLS + col) * OP + d);
      ll = fmaf(f, s_l[w * COLS + col], ll);
      a.x = fmaf(f, v.x, a.x);
      a.y = fmaf(f, v.y, a.y);
      a.z = fmaf(f, v.z, a.z);
      a.w = fmaf(f, v.w, a.w);
    }
    if (p.n_split == 1) {
      const float r = ll == 0.f ? 0.f : 1.0f / ll;
      const int cc = col0 + col, qi = cc / p.g, hh = cc - qi * p.g;
      __nv_bfloat16* dst = p.o + b * p.ob + qi * p.on + static_cast<int64_t>(hk * p.g + hh) * p.oh + d;
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(a.x * r, a.y * r), pack_bf16(a.z * r, a.w * r));
    } else {
      const int64_t piece = (static_cast<int64_t>(unit) * p.n_split + split) * COLS + col;
      const int64_t pieces = static_cast<int64_t>(gridDim.x) * COLS;
      *reinterpret_cast<float4*>(p.ws + piece * D + d) = a;
      if (d == 0) *reinterpret_cast<float2*>(p.ws + pieces * D + piece * 2) = make_float2(mm, ll);
    }
  }
}

// Joins the pieces of split sequences, in their order: one warp per (batch, column).
template <int D>
__global__ void __launch_bounds__(128) attn_kv4_join_kernel(const __grid_constant__ Kv4AttnParams p, const int cols, const int64_t pieces) {
  const int lane = threadIdx.x & 31;
  const int columns = p.n * p.g;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (item >= static_cast<int64_t>(p.B) * p.Hk * columns) return;
  const int bh = static_cast<int>(item / columns), cc = static_cast<int>(item - static_cast<int64_t>(bh) * columns);
  const int b = bh / p.Hk, hk = bh - b * p.Hk, chunk = cc / cols;
  int len = p.lengths[b];
  len = len < 0 ? 0 : min(len, p.max_len);
  int n = (len + p.split_len - 1) / p.split_len;
  if (n < 1) n = 1;
  const int64_t piece0 = (static_cast<int64_t>(bh) * p.col_chunks + chunk) * p.n_split * cols + (cc - chunk * cols);
  const float2* ml = reinterpret_cast<const float2*>(p.ws + pieces * D);
  float mm = -INFINITY;
  for (int s = lane; s < n; s += 32) mm = fmaxf(mm, ml[piece0 + static_cast<int64_t>(s) * cols].x);
#pragma unroll
  for (int d = 16; d; d >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, d));
  if (mm == -INFINITY) n = 0;
  float ll = 0.f;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  const bool live = lane * 4 < D;
#pragma unroll 4
  for (int s = 0; s < n; ++s) {
    const int64_t piece = piece0 + static_cast<int64_t>(s) * cols;
    const float2 x = ml[piece];
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (live) v = *reinterpret_cast<const float4*>(p.ws + piece * D + lane * 4);
    const float f = ak_ex2(x.x - mm);                            // 0 for a piece in which this column sees nothing
    ll = fmaf(f, x.y, ll);
    a.x = fmaf(f, v.x, a.x);
    a.y = fmaf(f, v.y, a.y);
    a.z = fmaf(f, v.z, a.z);
    a.w = fmaf(f, v.w, a.w);
  }
  const float r = ll == 0.f ? 0.f : 1.0f / ll;
  const int qi = cc / p.g, hh = cc - qi * p.g;
  if (live)
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
  auto kern = attn_kv4_kernel<D, G, NT>;
  constexpr size_t smem = ak_smem<D, G, NT>();
  cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), smem);
  if (e != cudaSuccess) return e;
  const int64_t grid = static_cast<int64_t>(p.B) * p.Hk * p.col_chunks * p.n_split;
  kern<<<static_cast<unsigned>(grid), AK_THREADS, smem, s>>>(p);
  e = cudaGetLastError();
  if (e != cudaSuccess || p.n_split == 1) return e;
  const int64_t items = static_cast<int64_t>(p.B) * p.Hk * p.n * p.g;
  attn_kv4_join_kernel<D><<<static_cast<unsigned>((items + 3) / 4), 128, 0, s>>>(p, 8 * NT, grid * 8 * NT);
  return cudaGetLastError();
}

template <int D, int G>
cudaError_t ak_cols(const Kv4AttnParams& p, cudaStream_t s) {
  return attn_kv4_cols(p.n * p.g) == 8 ? ak_run<D, G, 1>(p, s) : ak_run<D, G, 2>(p, s);
}
}  // namespace

int attn_kv4_resident(int head_dim, int group, int cols) { return cols == 8 ? 4 : 3; }

cudaError_t launch_attn_kv4(const Kv4AttnParams& p, int D, int G, int num_sms, cudaStream_t s) {
  if (D == 64) return G == 32 ? ak_cols<64, 32>(p, s) : ak_cols<64, 64>(p, s);
  if (D == 96) return ak_cols<96, 32>(p, s);
  return G == 32 ? ak_cols<128, 32>(p, s) : G == 64 ? ak_cols<128, 64>(p, s) : ak_cols<128, 128>(p, s);
}

}  // namespace gc
