// Keys and values into the paged 4-bit cache, and back as the values it holds.
//
// Both directions are bound by memory, if the work per element stays below about a dozen instructions.  A thread takes
// sixteen (writing) or eight (reading) consecutive elements of a few rows, all of whose loads are in flight together.
// Writing: the 2 / 4 / 8 threads of a group reduce minimum and maximum with shuffles, and each writes 64 bits of codes; the
// first of a group writes its (lo, scale).  Reading is the reverse.  Keys and values are the two halves of the grid's y dimension.
//
// The codes are decided on exact quotients.  n = rne((x - lo) * (1 / scale)) is right unless x lies next to a border between
// two codes, which the remainder x - lo - n scale tells: it is exact to 2^-20 of a scale, so only where it comes within 2^-16 of
// half a scale does the second look follow, which keeps x - lo as an exact sum of two floats and compares it with the borders
// (n -+ 1/2) scale, exact in fp32 themselves (a bf16 scale has 8 significant bits, 2 n +- 1 at most 5).
// Measured: 24000 tokens x 8 heads of 128, bf16, written 38 us (126 MB, 3.3 TB/s: bound by about 350 instructions for a thread's sixteen
// elements; 27 without the second look), read back 24 us (5.2 TB/s); 65000 tokens read 59 us (5.7 TB/s).
#include "ptx.cuh"
#include "serving.cuh"

namespace gc {

namespace {
constexpr int KV_THREADS = 256;

struct Kv4Params {
  gc_heads_t x[2];             // rows of keys, of values
  uint8_t* codes[2];
  uint32_t* params[2];
  const int64_t* slots;
  int64_t num_slots;
  uint32_t rows, heads;        // rows: tokens * heads
  uint32_t heads_mul, heads_shift;   // row / heads = (row * heads_mul) >> (32 + heads_shift)
  int page_shift;
  bool zeros;                  // reading: rows of no slot are zero (else left as they were)
  uint32_t* status;
};

// token and head of a row
__device__ __forceinline__ void split_row(const Kv4Params& p, uint32_t row, uint32_t* t, uint32_t* h) {
  *t = p.heads == 1 ? row : static_cast<uint32_t>((static_cast<uint64_t>(row) * p.heads_mul >> 32) >> p.heads_shift);
  *h = row - *t * p.heads;
}

// x - y exactly, as hi + lo (the two-term difference of Knuth)
__device__ __forceinline__ void exact_diff(float x, float y, float* hi, float* lo) {
  const float h = __fsub_rn(x, y);
  const float bb = __fsub_rn(h, x);
  *hi = h;
  *lo = __fsub_rn(__fsub_rn(x, __fsub_rn(h, bb)), __fadd_rn(y, bb));
}
// sign of (hi + lo) - b, exactly enough: where the first difference is inexact, it outweighs lo by far
__device__ __forceinline__ float minus_border(float hi, float lo, float b) { return __fadd_rn(__fsub_rn(hi, b), lo); }

__device__ __forceinline__ float bf16_down(float x) {       // the largest bf16 <= x, x finite
  const uint32_t u = __float_as_uint(x);
  uint32_t c = u & 0xffff0000u;
  if (c != u && (u >> 31)) c += 0x10000u;
  return __uint_as_float(c);
}

// (lo, scale) of a group from its minimum and maximum
__device__ __forceinline__ void group_params(float mn, float mx, float* lo_out, float* scale_out) {
  const float lo = bf16_down(mn);
  float dh, dl;
  exact_diff(mx, lo, &dh, &dl);
  // the smallest bf16 s >= d / 15, i.e. 15 s >= d: 15 s is exact (4 + 8 bits), the first guess one step off at most
  float s = -bf16_down(-(dh * (1.0f / 15.0f)));
  if (minus_border(dh, dl, 15.0f * s) > 0.0f) s = __uint_as_float(__float_as_uint(s) + 0x10000u);
  const float below = __uint_as_float(__float_as_uint(s) - 0x10000u);
  if (s > 0.0f && minus_border(dh, dl, 15.0f * below) <= 0.0f) s = below;
  *lo_out = lo;
  *scale_out = s;
}

// inv: about 1 / scale, or 0 where that leaves fp32
__device__ __forceinline__ uint32_t code_of(float x, float lo, float scale, float inv) {
  float dh, dl;
  exact_diff(x, lo, &dh, &dl);
  float n = fminf(rintf(inv > 0.0f ? dh * inv : __fdiv_rn(dh, scale)), 15.0f);
  const float up = minus_border(dh, dl, __fmul_rn(n + 0.5f, scale)), down = minus_border(dh, dl, __fmul_rn(n - 0.5f, scale));
  const bool odd = (__float_as_uint(n + 12582912.0f) & 1u) != 0;
  if (up > 0.0f || (up == 0.0f && odd)) n += 1.0f;
  else if (down < 0.0f || (down == 0.0f && odd)) n -= 1.0f;
  return __float_as_uint(fminf(fmaxf(n, 0.0f), 15.0f) + 12582912.0f) & 15u;
}

// Sixteen elements as they lie in memory.
template <typename T>
struct Raw {
  uint32_t w[4 * sizeof(T)];
};
template <typename T, bool VEC>
__device__ __forceinline__ Raw<T> load16(const T* x) {
  Raw<T> r;
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)); ++i) {
      const uint4 u = reinterpret_cast<const uint4*>(x)[i];
      r.w[4 * i] = u.x; r.w[4 * i + 1] = u.y; r.w[4 * i + 2] = u.z; r.w[4 * i + 3] = u.w;
    }
  } else if constexpr (sizeof(T) == 2) {
    const uint16_t* s = reinterpret_cast<const uint16_t*>(x);
#pragma unroll
    for (int i = 0; i < 8; ++i) r.w[i] = s[2 * i] | static_cast<uint32_t>(s[2 * i + 1]) << 16;
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) r.w[i] = __float_as_uint(x[i]);
  }
  return r;
}
template <typename T>
__device__ __forceinline__ float element(const Raw<T>& r, int i) {
  if constexpr (sizeof(T) == 2) return __uint_as_float(i & 1 ? r.w[i >> 1] & 0xffff0000u : r.w[i >> 1] << 16);
  else return __uint_as_float(r.w[i]);
}
// the same with an index known only at run time, without spilling the words
template <typename T>
__device__ __forceinline__ float pick(const Raw<T>& r, int i) {
  constexpr int N = 4 * sizeof(T);
  const int k = sizeof(T) == 2 ? i >> 1 : i;
  uint32_t w = r.w[0];
#pragma unroll
  for (int e = 1; e < N; ++e) w = k == e ? r.w[e] : w;
  if constexpr (sizeof(T) == 2) w = i & 1 ? w & 0xffff0000u : w << 16;
  return __uint_as_float(w);
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// Minimum and maximum of the elements, NaN if there is one among them.
template <typename T>
__device__ __forceinline__ void range16(const Raw<T>& r, float* mn, float* mx) {
  if constexpr (sizeof(T) == 2) {
    __nv_bfloat162 a = *reinterpret_cast<const __nv_bfloat162*>(&r.w[0]), b = a;
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      a = __hmin2_nan(a, *reinterpret_cast<const __nv_bfloat162*>(&r.w[i]));
      b = __hmax2_nan(b, *reinterpret_cast<const __nv_bfloat162*>(&r.w[i]));
    }
    *mn = min_nan(__low2float(a), __high2float(a));
    *mx = max_nan(__low2float(b), __high2float(b));
  } else {
    *mn = *mx = __uint_as_float(r.w[0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) {
      *mn = min_nan(*mn, __uint_as_float(r.w[i]));
      *mx = max_nan(*mx, __uint_as_float(r.w[i]));
    }
  }
}
// Two fp32 operations in one instruction, each rounded on its own.
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float* a, float* b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(*a), "=f"(*b) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
}  // namespace

// ITEMS rows per thread, a block's rows apart
template <typename T, int D, int G, bool VEC>
__global__ void __launch_bounds__(KV_THREADS) kv4_append_kernel(const __grid_constant__ Kv4Params p) {
  constexpr int LANES = D / 16, GL = G / 16, NG = D / G, ITEMS = 2, ROWS = KV_THREADS / LANES;
  wait_for_predecessor();
  const int which = blockIdx.y, j = threadIdx.x % LANES;
  const uint32_t row0 = blockIdx.x * (ROWS * ITEMS) + threadIdx.x / LANES;
  const gc_heads_t& x = p.x[which];
  Raw<T> raw[ITEMS];
  int64_t slot[ITEMS];
  uint32_t head[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const uint32_t row = min(row0 + i * ROWS, p.rows - 1);       // surplus threads repeat the last row, and write nothing
    uint32_t t;
    split_row(p, row, &t, &head[i]);
    raw[i] = load16<T, VEC>(static_cast<const T*>(x.data) + t * x.token_stride + head[i] * x.head_stride + j * 16);
    slot[i] = p.slots[t];
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    float mn, mx;
    range16(raw[i], &mn, &mx);
#pragma unroll
    for (int d = GL / 2; d; d >>= 1) {
      mn = min_nan(mn, __shfl_xor_sync(0xffffffffu, mn, d));
      mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    }
    if (threadIdx.x >= ROWS * LANES || row0 + i * ROWS >= p.rows || slot[i] < 0) continue;
    if (slot[i] >= p.num_slots) {
      report(p.status, DEV_BAD_SLOT);
      continue;
    }
    uint32_t word[2] = {0, 0}, pw = 0x7fc07fc0u;                 // a group that cannot be held: NaN
    if (mn >= -3.402823466e38f && mx <= 3.402823466e38f) {
      float lo, scale;
      group_params(mn, mx, &lo, &scale);
      if (scale <= 3.402823466e38f) {
        pw = (__float_as_uint(lo) >> 16) | __float_as_uint(scale);
        uint32_t border = 0;                                     // elements that need the second look
        float inv = 0.0f;
        if (scale > 0x1p-100f) {                                 // every product below is a normal number
          // (the estimate's quotient is off by 2^-22 of at most 15: well within `near` of a border where it picks the wrong side)
          asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(scale));
          const float half = 0.5f * scale, near = 0x1p-16f * scale;
          constexpr float magic = 12582912.0f;                   // 1.5 * 2^23: adding it rounds to a whole number, ties to even
          const uint64_t nlo2 = pair(-lo, -lo), inv2 = pair(inv, inv), m2 = pair(magic, magic), minus2 = pair(-1.0f, -1.0f);
          const uint64_t s2 = pair(scale, scale), sixteen2 = pair(16.0f, 16.0f);
          uint64_t sum[4];                                       // two by two: codes of elements e, e + 2, e + 4, e + 6 as digits
#pragma unroll
          for (int e = 14; e >= 0; e -= 2) {
            const uint64_t d = add2(pair(element(raw[i], e), element(raw[i], e + 1)), nlo2);
            const uint64_t nn = fma2(fma2(d, inv2, m2), minus2, m2);                   // - n
            float r0, r1;
            unpair(fma2(nn, s2, d), &r0, &r1);                   // d - n scale
            if (fabsf(fabsf(r0) - half) <= near) border |= 1u << e;
            if (fabsf(fabsf(r1) - half) <= near) border |= 2u << e;
            sum[e >> 2] = (e & 2) ? nn : fma2(sum[e >> 2], sixteen2, nn);
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {                          // elements 8 h .. 8 h + 7: digits of base 16, even and odd ones
            float a0, a1, b0, b1;
            unpair(sum[2 * h], &a0, &a1);
            unpair(sum[2 * h + 1], &b0, &b1);
            // - (code[0] + 16 code[2]), of code[1], code[3], of code[4], code[6], of code[5], code[7]
            const uint32_t ev = __float_as_uint(8388608.0f - a0) & 0xffu, od = __float_as_uint(8388608.0f - a1) & 0xffu;
            const uint32_t ev2 = __float_as_uint(8388608.0f - b0) & 0xffu, od2 = __float_as_uint(8388608.0f - b1) & 0xffu;
            const uint32_t lo4 = (ev & 15u) | (od & 15u) << 4 | (ev >> 4) << 8 | (od >> 4) << 12;
            const uint32_t hi4 = (ev2 & 15u) | (od2 & 15u) << 4 | (ev2 >> 4) << 8 | (od2 >> 4) << 12;
            word[h] = lo4 | hi4 << 16;
          }
        } else if (scale > 0.0f) {
          border = 0xffffu;
        }
        while (border) {                                         // (ties are not rare in bf16: one element in 200)
          const int e = __ffs(border) - 1, sh = 4 * (e & 7);
          border &= border - 1;
          const float x = pick(raw[i], e), d = x - lo;
          const uint32_t was = (e < 8 ? word[0] : word[1]) >> sh & 15u;
          const float r = fmaf(8388608.0f - __uint_as_float(was | 0x4b000000u), scale, d);       // d - code scale, exact here
          uint32_t is = was;
          if (fabsf(r) == 0.5f * scale && d + lo == x && x - d == lo) {
            if (was & 1u) is = r > 0.0f ? was + 1 : was - 1;     // a tie of exact numbers: the even one
          } else {
            is = code_of(x, lo, scale, inv);
          }
          const uint32_t flip = (was ^ is) << sh;
          word[0] ^= e < 8 ? flip : 0u;
          word[1] ^= e < 8 ? 0u : flip;
        }
      }
    }
    const int64_t page = slot[i] >> p.page_shift;
    const int64_t r = ((page * p.heads + head[i]) << p.page_shift) + (slot[i] & ((1 << p.page_shift) - 1));
    *reinterpret_cast<uint2*>(p.codes[which] + r * (D / 2) + j * 8) = make_uint2(word[0], word[1]);
    if (j % GL == 0) p.params[which][r * NG + j / GL] = pw;
  }
}

template <typename T, int D, int G, bool VEC>
__global__ void __launch_bounds__(KV_THREADS) kv4_read_kernel(const __grid_constant__ Kv4Params p) {
  constexpr int LANES = D / 8, GL = G / 8, NG = D / G, ITEMS = 4, ROWS = KV_THREADS / LANES;
  wait_for_predecessor();
  const int which = blockIdx.y, j = threadIdx.x % LANES;
  const uint32_t row0 = blockIdx.x * (ROWS * ITEMS) + threadIdx.x / LANES;
  const gc_heads_t& x = p.x[which];
  if (threadIdx.x >= ROWS * LANES) return;
  int64_t slot[ITEMS];
  uint32_t t[ITEMS], h[ITEMS], word[ITEMS], pw[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    split_row(p, min(row0 + i * ROWS, p.rows - 1), &t[i], &h[i]);
    slot[i] = row0 + i * ROWS < p.rows ? p.slots[t[i]] : -1;
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    word[i] = pw[i] = 0;
    if (slot[i] >= p.num_slots) {
      report(p.status, DEV_BAD_SLOT);
      slot[i] = -1;
    }
    if (slot[i] < 0) continue;
    const int64_t page = slot[i] >> p.page_shift;
    const int64_t r = ((page * p.heads + h[i]) << p.page_shift) + (slot[i] & ((1 << p.page_shift) - 1));
    word[i] = *reinterpret_cast<const uint32_t*>(p.codes[which] + r * (D / 2) + j * 4);
    pw[i] = p.params[which][r * NG + j / GL];
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    if (slot[i] < 0 && !(p.zeros && row0 + i * ROWS < p.rows)) continue;       // (code and parameters of no slot are zeros)
    T* dst = static_cast<T*>(x.data) + t[i] * x.token_stride + h[i] * x.head_stride + j * 8;
    if constexpr (sizeof(T) == 2) {
      // pairs (0,4), (1,5), (2,6), (3,7): 128 + code, minus 128, times scale plus lo in one rounding
      const uint32_t lo2 = __byte_perm(pw[i], 0, 0x1010), sc2 = __byte_perm(pw[i], 0, 0x3232);
      const uint32_t m128 = 0xc300c300u;
      uint32_t v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t n = ((word[i] >> (4 * e)) & 0x000f000fu) | 0x43004300u;
        const __nv_bfloat162 c = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&n), *reinterpret_cast<const __nv_bfloat162*>(&m128));
        const __nv_bfloat162 f = __hfma2(c, *reinterpret_cast<const __nv_bfloat162*>(&sc2), *reinterpret_cast<const __nv_bfloat162*>(&lo2));
        v[e] = *reinterpret_cast<const uint32_t*>(&f);
      }
      const uint32_t w[4] = {__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410), __byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632)};
      if constexpr (VEC) {
        *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) reinterpret_cast<uint16_t*>(dst)[e] = static_cast<uint16_t>(w[e >> 1] >> (16 * (e & 1)));
      }
    } else {
      const float lo = __uint_as_float(pw[i] << 16), scale = __uint_as_float(pw[i] & 0xffff0000u);
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)                                // the code as a float: 2^23 + code, minus 2^23; the product is exact
        v[e] = fmaf(__uint_as_float(((word[i] >> (4 * e)) & 15u) | 0x4b000000u) - 8388608.0f, scale, lo);
      if constexpr (VEC) {
        reinterpret_cast<float4*>(dst)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(dst)[1] = make_float4(v[4], v[5], v[6], v[7]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) dst[e] = static_cast<T>(v[e]);
      }
    }
  }
}

namespace {
bool vec_heads(const gc_heads_t& h, int esz) {
  return reinterpret_cast<uintptr_t>(h.data) % 16 == 0 && (h.token_stride * esz) % 16 == 0 && (h.head_stride * esz) % 16 == 0;
}

template <bool READ, typename T, int D, int G>
cudaError_t run(const Kv4Params& p, bool vec, cudaStream_t s) {
  const uint32_t per = READ ? KV_THREADS / (D / 8) * 4 : KV_THREADS / (D / 16) * 2;
  const uint32_t gx = (p.rows + per - 1) / per;
  const dim3 grid(gx, 2);
  if constexpr (READ) return launch_following(vec ? kv4_read_kernel<T, D, G, true> : kv4_read_kernel<T, D, G, false>, grid, KV_THREADS, 0, s, p);
  else return launch_following(vec ? kv4_append_kernel<T, D, G, true> : kv4_append_kernel<T, D, G, false>, grid, KV_THREADS, 0, s, p);
}

template <bool READ, typename T>
cudaError_t dispatch(const Kv4Params& p, int D, int G, bool vec, cudaStream_t s) {
  if (D == 64) return G == 32 ? run<READ, T, 64, 32>(p, vec, s) : run<READ, T, 64, 64>(p, vec, s);
  if (D == 96) return run<READ, T, 96, 32>(p, vec, s);
  return G == 32 ? run<READ, T, 128, 32>(p, vec, s) : G == 64 ? run<READ, T, 128, 64>(p, vec, s) : run<READ, T, 128, 128>(p, vec, s);
}

template <bool READ>
cudaError_t launch(const gc_kv4_cache_t& c, int dtype, int64_t tokens, const gc_heads_t& k, const gc_heads_t& v, const int64_t* slots,
                   bool zeros, cudaStream_t s) {
  Kv4Params p = {};
  p.x[0] = k; p.x[1] = v;
  p.codes[0] = static_cast<uint8_t*>(c.k_codes); p.codes[1] = static_cast<uint8_t*>(c.v_codes);
  p.params[0] = static_cast<uint32_t*>(c.k_params); p.params[1] = static_cast<uint32_t*>(c.v_params);
  p.slots = slots;
  p.num_slots = c.num_pages * c.page_size;
  p.rows = static_cast<uint32_t>(tokens * c.kv_heads);
  p.heads = c.kv_heads;
  // row / heads for row < 2^31: heads_mul = ceil(2^(32 + shift) / heads), shift = ceil(log2 heads) - 1, fits 32 bits
  while ((2u << p.heads_shift) < p.heads) ++p.heads_shift;
  p.heads_mul = static_cast<uint32_t>(((1ull << (32 + p.heads_shift)) + p.heads - 1) / p.heads);
  while ((1 << p.page_shift) < c.page_size) ++p.page_shift;
  p.zeros = zeros;
  p.status = c.status;
  const int esz = dtype == GC_F32 ? 4 : 2;
  const bool vec = vec_heads(k, esz) && vec_heads(v, esz);
  return dtype == GC_F32 ? dispatch<READ, float>(p, c.head_dim, c.group, vec, s)
                         : dispatch<READ, __nv_bfloat16>(p, c.head_dim, c.group, vec, s);
}
}  // namespace

cudaError_t launch_kv4_append(const gc_kv4_cache_t& c, int dtype, int64_t tokens, const gc_heads_t& k, const gc_heads_t& v,
                              const int64_t* slots, cudaStream_t s) {
  return launch<false>(c, dtype, tokens, k, v, slots, false, s);
}
cudaError_t launch_kv4_read(const gc_kv4_cache_t& c, int dtype, int64_t tokens, const gc_heads_t& k, const gc_heads_t& v,
                            const int64_t* slots, bool zeros, cudaStream_t s) {
  return launch<true>(c, dtype, tokens, k, v, slots, zeros, s);
}

}  // namespace gc
