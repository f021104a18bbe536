// Keys and values into the paged 4-bit cache, and back as the values it holds.
//
// Both directions are bound by memory.  Writing: a thread holds eight consecutive elements of a row, the 4 / 8 / 16
// threads of a group reduce minimum and maximum with shuffles, and each writes one 32-bit word of codes; the first of a
// group writes its (lo, scale).  Reading is the reverse.  Keys and values are the two halves of the grid's y dimension.
//
// The codes are decided on exact quotients.  d = x - lo is kept as an exact sum of two floats (dh + dl); the candidate
// n = rne(dh * (1 / scale)) is within one of the answer, and the borders (n -+ 1/2) * scale are exact in fp32 (a bf16
// scale has 8 significant bits, 2 n +- 1 at most 5), so d is compared with them without rounding.
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
  int64_t tokens, num_slots, items;   // items: tokens * heads * D / 8
  int heads, page_shift;
  uint32_t* status;
};

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
  // the smallest bf16 s >= d / 15, i.e. 15 s >= d: 15 s is exact (4 + 8 bits)
  float s = -bf16_down(-__fdiv_rn(dh, 15.0f));
  if (minus_border(dh, dl, 15.0f * s) > 0.0f) s = __uint_as_float(__float_as_uint(s) + 0x10000u);
  const float below = __uint_as_float(__float_as_uint(s) - 0x10000u);
  if (s > 0.0f && minus_border(dh, dl, 15.0f * below) <= 0.0f) s = below;
  *lo_out = lo;
  *scale_out = s;
}

__device__ __forceinline__ uint32_t code_of(float x, float lo, float scale, float inv) {
  float dh, dl;
  exact_diff(x, lo, &dh, &dl);
  // (the reciprocal of a scale near the smallest numbers overflows: divide there)
  float n = fminf(rintf(inv <= 3.402823466e38f ? dh * inv : __fdiv_rn(dh, scale)), 15.0f);
  const float up = minus_border(dh, dl, __fmul_rn(n + 0.5f, scale)), down = minus_border(dh, dl, __fmul_rn(n - 0.5f, scale));
  const bool odd = (static_cast<int>(n) & 1) != 0;
  if (up > 0.0f || (up == 0.0f && odd)) n += 1.0f;
  else if (down < 0.0f || (down == 0.0f && odd)) n -= 1.0f;
  return static_cast<uint32_t>(fminf(fmaxf(n, 0.0f), 15.0f));
}

template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* x, float (&v)[8]) {
  if constexpr (VEC && sizeof(T) == 2) {
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(x));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else if constexpr (VEC) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(x)), b = __ldg(reinterpret_cast<const float4*>(x) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(x[i]);
  }
}
}  // namespace

template <typename T, int D, int G, bool VEC>
__global__ void __launch_bounds__(KV_THREADS) kv4_append_kernel(const __grid_constant__ Kv4Params p) {
  constexpr int LANES = D / 8, GL = G / 8, NG = D / G;
  const int which = blockIdx.y;
  const gc_heads_t& x = p.x[which];
  const int64_t item = static_cast<int64_t>(blockIdx.x) * KV_THREADS + threadIdx.x;
  const bool live = item < p.items;
  const int64_t row = live ? item / LANES : 0;
  const int j = live ? static_cast<int>(item - row * LANES) : 0;
  const int64_t t = row / p.heads;
  const int h = static_cast<int>(row - t * p.heads);
  float v[8];
  load8<T, VEC>(static_cast<const T*>(x.data) + t * x.token_stride + h * x.head_stride + j * 8, v);
  const int64_t slot = __ldg(p.slots + t);
  float mn = v[0], mx = v[0];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    mn = fminf(mn, v[i]);
    mx = fmaxf(mx, v[i]);
    bad |= !(fabsf(v[i]) <= 3.402823466e38f);
  }
  int badi = bad;
#pragma unroll
  for (int d = GL / 2; d; d >>= 1) {
    mn = fminf(mn, __shfl_xor_sync(0xffffffffu, mn, d));
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    badi |= __shfl_xor_sync(0xffffffffu, badi, d);
  }
  if (!live || slot < 0) return;
  if (slot >= p.num_slots) {
    report(p.status, DEV_BAD_SLOT);
    return;
  }
  float lo, scale;
  group_params(mn, mx, &lo, &scale);
  uint32_t word = 0, pw;
  if (badi || !(scale <= 3.402823466e38f)) {
    pw = 0x7fc07fc0u;                                              // the group is held as NaN
  } else {
    if (scale > 0.0f) {
      const float inv = 1.0f / scale;
#pragma unroll
      for (int i = 0; i < 8; ++i) word |= code_of(v[i], lo, scale, inv) << (4 * i);
    }
    pw = (__float_as_uint(lo) >> 16) | __float_as_uint(scale);
  }
  const int64_t page = slot >> p.page_shift;
  const int64_t r = (((page * p.heads + h) << p.page_shift) + (slot & ((1 << p.page_shift) - 1)));
  *reinterpret_cast<uint32_t*>(p.codes[which] + r * (D / 2) + j * 4) = word;
  if (j % GL == 0) p.params[which][r * NG + j / GL] = pw;
}

// ITEMS groups of eight elements per thread, a block's width apart, so that their loads are in flight together
template <typename T, int D, int G, bool VEC>
__global__ void __launch_bounds__(KV_THREADS) kv4_read_kernel(const __grid_constant__ Kv4Params p) {
  constexpr int LANES = D / 8, GL = G / 8, NG = D / G, ITEMS = 4;
  const int which = blockIdx.y;
  const gc_heads_t& x = p.x[which];
  const int64_t item0 = static_cast<int64_t>(blockIdx.x) * (KV_THREADS * ITEMS) + threadIdx.x;
  uint32_t word[ITEMS], pw[ITEMS];
  T* dst[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int64_t item = item0 + i * KV_THREADS;
    dst[i] = nullptr;
    word[i] = pw[i] = 0;
    if (item >= p.items) continue;
    const int64_t row = item / LANES;
    const int j = static_cast<int>(item - row * LANES);
    const int64_t t = row / p.heads;
    const int h = static_cast<int>(row - t * p.heads);
    const int64_t slot = __ldg(p.slots + t);
    if (slot < 0) continue;
    if (slot >= p.num_slots) {
      report(p.status, DEV_BAD_SLOT);
      continue;
    }
    const int64_t page = slot >> p.page_shift;
    const int64_t r = (((page * p.heads + h) << p.page_shift) + (slot & ((1 << p.page_shift) - 1)));
    word[i] = __ldg(reinterpret_cast<const uint32_t*>(p.codes[which] + r * (D / 2) + j * 4));
    pw[i] = __ldg(p.params[which] + r * NG + j / GL);
    dst[i] = static_cast<T*>(x.data) + t * x.token_stride + h * x.head_stride + j * 8;
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    if (!dst[i]) continue;
    const float lo = __uint_as_float(pw[i] << 16), scale = __uint_as_float(pw[i] & 0xffff0000u);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fmaf(static_cast<float>((word[i] >> (4 * e)) & 15u), scale, lo);   // the product is exact
    if constexpr (VEC && sizeof(T) == 2) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
        w[e] = *reinterpret_cast<const uint32_t*>(&b);
      }
      *reinterpret_cast<uint4*>(dst[i]) = make_uint4(w[0], w[1], w[2], w[3]);
    } else if constexpr (VEC) {
      reinterpret_cast<float4*>(dst[i])[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(dst[i])[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) dst[i][e] = static_cast<T>(v[e]);
    }
  }
}

namespace {
bool vec_heads(const gc_heads_t& h, int esz) {
  return reinterpret_cast<uintptr_t>(h.data) % 16 == 0 && (h.token_stride * esz) % 16 == 0 && (h.head_stride * esz) % 16 == 0;
}

template <bool READ, typename T, int D, int G>
cudaError_t run(const Kv4Params& p, bool vec, cudaStream_t s) {
  const int64_t per = KV_THREADS * (READ ? 4 : 1);
  const int64_t gx = (p.items + per - 1) / per;
  if (gx > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(gx), 2);
  if constexpr (READ) {
    if (vec) kv4_read_kernel<T, D, G, true><<<grid, KV_THREADS, 0, s>>>(p);
    else kv4_read_kernel<T, D, G, false><<<grid, KV_THREADS, 0, s>>>(p);
  } else {
    if (vec) kv4_append_kernel<T, D, G, true><<<grid, KV_THREADS, 0, s>>>(p);
    else kv4_append_kernel<T, D, G, false><<<grid, KV_THREADS, 0, s>>>(p);
  }
  return cudaGetLastError();
}

template <bool READ, typename T>
cudaError_t dispatch(const Kv4Params& p, int D, int G, bool vec, cudaStream_t s) {
  if (D == 64) return G == 32 ? run<READ, T, 64, 32>(p, vec, s) : run<READ, T, 64, 64>(p, vec, s);
  if (D == 96) return run<READ, T, 96, 32>(p, vec, s);
  return G == 32 ? run<READ, T, 128, 32>(p, vec, s) : G == 64 ? run<READ, T, 128, 64>(p, vec, s) : run<READ, T, 128, 128>(p, vec, s);
}

template <bool READ>
cudaError_t launch(const gc_kv4_cache_t& c, int dtype, int64_t tokens, const gc_heads_t& k, const gc_heads_t& v, const int64_t* slots,
                   cudaStream_t s) {
  Kv4Params p = {};
  p.x[0] = k; p.x[1] = v;
  p.codes[0] = static_cast<uint8_t*>(c.k_codes); p.codes[1] = static_cast<uint8_t*>(c.v_codes);
  p.params[0] = static_cast<uint32_t*>(c.k_params); p.params[1] = static_cast<uint32_t*>(c.v_params);
  p.slots = slots;
  p.tokens = tokens;
  p.num_slots = c.num_pages * c.page_size;
  p.items = tokens * c.kv_heads * (c.head_dim / 8);
  p.heads = c.kv_heads;
  while ((1 << p.page_shift) < c.page_size) ++p.page_shift;
  p.status = c.status;
  const int esz = dtype == GC_F32 ? 4 : 2;
  const bool vec = vec_heads(k, esz) && vec_heads(v, esz);
  return dtype == GC_F32 ? dispatch<READ, float>(p, c.head_dim, c.group, vec, s)
                         : dispatch<READ, __nv_bfloat16>(p, c.head_dim, c.group, vec, s);
}
}  // namespace

cudaError_t launch_kv4_append(const gc_kv4_cache_t& c, int dtype, int64_t tokens, const gc_heads_t& k, const gc_heads_t& v,
                              const int64_t* slots, cudaStream_t s) {
  return launch<false>(c, dtype, tokens, k, v, slots, s);
}
cudaError_t launch_kv4_read(const gc_kv4_cache_t& c, int dtype, int64_t tokens, const gc_heads_t& k, const gc_heads_t& v,
                            const int64_t* slots, cudaStream_t s) {
  return launch<true>(c, dtype, tokens, k, v, slots, s);
}

}  // namespace gc
