// RMS norm of every query and key head and the rotation of its elements by position, one pass over the data.
//
//   y = x * rsqrt(mean(x^2) + eps) * w ;   (a, b) -> (a cos phi - b sin phi, b cos phi + a sin phi),  phi = pos * inv_freq[i]
//
// Bound by memory: every element is read once and written once, about 7 operations each.  The angles of a token are the
// same for all of its heads, so a CTA takes whole tokens and evaluates cos / sin once per (token, pair) into shared memory
// (the product pos * inv_freq and its reduction by multiples of 2 pi in fp64, since a far position times a frequency
// leaves fp32 no fraction).  Then a few lanes share a row, two 16-byte vectors each, chosen so that both halves of every
// pair are in one lane: vectors j and j + rot / 2, or two neighbours where pairs are interleaved.  A lane keeps its angles
// and weights in registers and walks the heads of its token, the next row's loads under way while it works on one.
// Rows that are not 16-byte aligned, or whose sizes do not come out in such vectors, take a second kernel, which hands the
// normalised row over in shared memory, where the other half of a pair is picked up.
// Measured: 8191 tokens x 40 heads of 128, bf16 (168 MB): 37.5 us = 4.5 TB/s (that second kernel: 66); 1537 x 32 of 64, fp32: 6.3 us
// (11.6); 16 tokens: 4.2 us, a launch and four dependent trips to memory.
#include "serving.cuh"

namespace gc {

namespace {
constexpr int QN_THREADS = 256;

struct QkParams {
  gc_heads_t q, k, q_out, k_out;
  const void* q_weight;
  const void* k_weight;
  const int64_t* positions;
  const float* inv_freq;
  int64_t tokens;
  int q_heads, rows;           // rows of a token: q_heads + k_heads
  int D, half, interleaved, norm;
  float eps, factor;
  int tb;                      // tokens per CTA
  int rows_per_cta;            // rows of each token one CTA takes (grid.y parts of them)
  int log_l;                   // log2 of the lanes per row
};

template <typename T>
__device__ __forceinline__ float to_f(T x);
template <>
__device__ __forceinline__ float to_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ float from_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// 16 bytes of rounded elements
template <typename T>
__device__ __forceinline__ uint4 pack16(const float* y) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    } else {
      w[i] = __float_as_uint(y[i]);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// cos and sin of pos * f, both times `factor`.  2 pi = TWO_PI_HI + TWO_PI_LO to about 106 bits.
__device__ __forceinline__ void turn_of(int64_t pos, float f, float factor, float* c, float* s) {
  constexpr double TWO_PI_HI = 6.283185307179586232, TWO_PI_LO = 2.4492935982947064e-16;
  const double phi = static_cast<double>(pos) * static_cast<double>(f);
  const double n = rint(phi * (1.0 / TWO_PI_HI));
  const float r = static_cast<float>(fma(-n, TWO_PI_LO, fma(-n, TWO_PI_HI, phi)));
  float sn, cs;
  sincosf(r, &sn, &cs);
  *c = cs * factor;
  *s = sn * factor;
}
}  // namespace

// T: element type, W: consecutive elements per lane (16 bytes, or 1), CH: chunks of L * W elements per row
template <typename T, int W, int CH>
__global__ void __launch_bounds__(QN_THREADS) qk_norm_rope_kernel(const __grid_constant__ QkParams p) {
  extern __shared__ float4 smem4[];
  wait_for_predecessor();
  const int L = 1 << p.log_l, slots = QN_THREADS >> p.log_l;
  float* s_row = reinterpret_cast<float*>(smem4);                        // [slots][D rounded up to 4]
  const int pitch = (p.D + 3) & ~3, tpitch = (p.half + 3) & ~3;
  float* s_cos = s_row + slots * pitch;                                  // [tb][half]
  float* s_sin = s_cos + p.tb * tpitch;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * p.tb;
  const int nt = static_cast<int>(p.tokens - t0 < p.tb ? p.tokens - t0 : p.tb);
  const int r0 = blockIdx.y * p.rows_per_cta;
  const int nr = p.rows - r0 < p.rows_per_cta ? p.rows - r0 : p.rows_per_cta;

  for (int i = threadIdx.x; i < nt * p.half; i += QN_THREADS) {
    const int t = i / p.half, j = i - t * p.half;
    turn_of(p.positions[t0 + t], p.inv_freq[j], p.factor, s_cos + t * tpitch + j, s_sin + t * tpitch + j);
  }
  __syncthreads();

  const int lane = threadIdx.x & (L - 1), slot = threadIdx.x >> p.log_l;
  float* row = s_row + slot * pitch;
  const int total = nt * nr, rot = 2 * p.half;
  const bool vec_pairs = W > 1 && p.half % W == 0;
  for (int base = 0; base < total; base += slots) {
    const int u = base + slot;
    const bool live = u < total;
    const int t = live ? u / nr : 0, h = live ? r0 + u - t * nr : 0;
    const bool is_q = h < p.q_heads;
    const gc_heads_t& src = is_q ? p.q : p.k;
    const gc_heads_t& dst = is_q ? p.q_out : p.k_out;
    const int hh = is_q ? h : h - p.q_heads;
    const T* x = static_cast<const T*>(src.data) + (t0 + t) * src.token_stride + hh * src.head_stride;
    T* o = static_cast<T*>(dst.data) + (t0 + t) * dst.token_stride + hh * dst.head_stride;
    const T* w = static_cast<const T*>(is_q ? p.q_weight : p.k_weight);
    float y[CH][W];
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int e = (c * L + lane) * W;
      if (live && e < p.D) {
        if constexpr (W > 1) {
          const uint4 v = *reinterpret_cast<const uint4*>(x + e);
          const T* ve = reinterpret_cast<const T*>(&v);
#pragma unroll
          for (int i = 0; i < W; ++i) y[c][i] = to_f<T>(ve[i]);
        } else {
          y[c][0] = to_f<T>(x[e]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < W; ++i) y[c][i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < W; ++i) sum = fmaf(y[c][i], y[c][i], sum);
    }
    if (p.norm) {
      for (int d = L >> 1; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      const float inv = rsqrtf(sum / static_cast<float>(p.D) + p.eps);
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int e = (c * L + lane) * W;
        if (live && e < p.D) {
          if (w) {
            if constexpr (W > 1) {
              const uint4 v = *reinterpret_cast<const uint4*>(w + e);
              const T* ve = reinterpret_cast<const T*>(&v);
#pragma unroll
              for (int i = 0; i < W; ++i) y[c][i] = y[c][i] * inv * to_f<T>(ve[i]);
            } else {
              y[c][0] = y[c][0] * inv * to_f<T>(w[e]);
            }
          } else {
#pragma unroll
            for (int i = 0; i < W; ++i) y[c][i] *= inv;
          }
        }
      }
    }
    const float* ct = s_cos + t * tpitch;
    const float* st = s_sin + t * tpitch;
    if (W > 1 && p.interleaved) {
      // both elements of a pair lie in the lane's own chunk
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int e = (c * L + lane) * W;
#pragma unroll
        for (int i = 0; i + 1 < W; i += 2) {
          if (e + i < rot) {
            const int j = (e + i) >> 1;
            const float a = y[c][i], b = y[c][i + 1], cs = ct[j], sn = st[j];
            y[c][i] = a * cs - b * sn;
            y[c][i + 1] = b * cs + a * sn;
          }
        }
      }
    } else if (rot) {
      __syncwarp();                                                      // the previous row has been read
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int e = (c * L + lane) * W;
        if (e < p.D) {
          if constexpr (W == 8) {
            *reinterpret_cast<float4*>(row + e) = make_float4(y[c][0], y[c][1], y[c][2], y[c][3]);
            *reinterpret_cast<float4*>(row + e + 4) = make_float4(y[c][4], y[c][5], y[c][6], y[c][7]);
          } else if constexpr (W == 4) {
            *reinterpret_cast<float4*>(row + e) = make_float4(y[c][0], y[c][1], y[c][2], y[c][3]);
          } else {
            row[e] = y[c][0];
          }
        }
      }
      __syncwarp();
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int e = (c * L + lane) * W;
        if (e < rot) {
          if (vec_pairs) {
            // half layout, the chunk on one side of the middle: partners and angles are vectors
            const bool low = e < p.half;
            const int j = low ? e : e - p.half, pe = low ? e + p.half : j;
#pragma unroll
            for (int i = 0; i < W; i += (W >= 4 ? 4 : 1)) {
              if constexpr (W >= 4) {
                const float4 b = *reinterpret_cast<const float4*>(row + pe + i);
                const float4 cs = *reinterpret_cast<const float4*>(ct + j + i);
                const float4 sn = *reinterpret_cast<const float4*>(st + j + i);
                const float g = low ? -1.f : 1.f;
                y[c][i] = fmaf(y[c][i], cs.x, g * b.x * sn.x);
                y[c][i + 1] = fmaf(y[c][i + 1], cs.y, g * b.y * sn.y);
                y[c][i + 2] = fmaf(y[c][i + 2], cs.z, g * b.z * sn.z);
                y[c][i + 3] = fmaf(y[c][i + 3], cs.w, g * b.w * sn.w);
              }
            }
          } else {
#pragma unroll
            for (int i = 0; i < W; ++i) {
              const int ee = e + i;
              if (ee < rot) {
                const bool low = p.interleaved ? !(ee & 1) : ee < p.half;
                const int j = p.interleaved ? ee >> 1 : (low ? ee : ee - p.half);
                const int pe = p.interleaved ? ee ^ 1 : (low ? ee + p.half : j);
                const float b = row[pe];
                y[c][i] = y[c][i] * ct[j] + (low ? -b : b) * st[j];
              }
            }
          }
        }
      }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int e = (c * L + lane) * W;
      if (live && e < p.D) {
        if constexpr (W > 1) {
          uint4 v;
          T* ve = reinterpret_cast<T*>(&v);
#pragma unroll
          for (int i = 0; i < W; ++i) ve[i] = from_f<T>(y[c][i]);
          *reinterpret_cast<uint4*>(o + e) = v;
        } else {
          o[e] = from_f<T>(y[c][0]);
        }
      }
    }
  }
}

// W: elements in 16 bytes.  L = 1 << log_l lanes per row, two vectors of W elements each (D / (2 W) lanes of them busy).
template <typename T, int W, bool INTERLEAVED>
__global__ void __launch_bounds__(QN_THREADS, 3) qk_norm_rope_pairs_kernel(const __grid_constant__ QkParams p) {
  extern __shared__ float4 smem4[];
  wait_for_predecessor();
  const int tpitch = (p.half + W - 1) / W * W;                   // angles of a token, padded to whole vectors
  float* s_cos = reinterpret_cast<float*>(smem4);
  float* s_sin = s_cos + p.tb * tpitch;
  // pair i of a lane: elements i of its two vectors, or neighbours in one of them
  auto turn = [](float (&y0)[W], float (&y1)[W], int i, float c, float s) {
    float& a = INTERLEAVED ? (i < W / 2 ? y0[(2 * i) % W] : y1[(2 * i) % W]) : y0[i];
    float& b = INTERLEAVED ? (i < W / 2 ? y0[(2 * i + 1) % W] : y1[(2 * i + 1) % W]) : y1[i];
    const float u = a, v = b;
    a = fmaf(u, c, -(v * s));
    b = fmaf(v, c, u * s);
  };
  const float inv_d = 1.0f / static_cast<float>(p.D);
  const int L = 1 << p.log_l, item = threadIdx.x & (L - 1);
  const int slot = threadIdx.x >> p.log_l, per_token = (QN_THREADS >> p.log_l) / p.tb;         // rows a token's slots take at a time
  const int t = slot / per_token, s0 = slot - t * per_token;
  const bool mine = 2 * W * item < p.D;                          // else a lane without elements, there for the shuffles
  // the two vectors, and the first angle
  const int low = p.half / W;                                    // vectors below the middle (not interleaved)
  const bool turns = INTERLEAVED || item < low;
  const int e0 = INTERLEAVED ? 2 * W * item : turns ? W * item : 2 * p.half + 2 * W * (item - low);
  const int e1 = !INTERLEAVED && turns ? p.half + W * item : e0 + W;
  const int angles = max(min(p.half - W * item, W), 0);          // pairs of this lane that turn (interleaved; else all or none)
  const int r0 = blockIdx.y * p.rows_per_cta, r1 = min(r0 + p.rows_per_cta, p.rows);
  // groups of tb tokens, a grid's width apart
  for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * p.tb; t0 < p.tokens; t0 += static_cast<int64_t>(gridDim.x) * p.tb) {
    const int nt = static_cast<int>(p.tokens - t0 < p.tb ? p.tokens - t0 : p.tb);
    const bool live_token = t < nt;
    if (mine && live_token) {                                      // the first rows on their way while the angles are evaluated
      const bool is_q = r0 + s0 < p.q_heads;
      const gc_heads_t& src = is_q ? p.q : p.k;
      const T* x = static_cast<const T*>(src.data) + (t0 + t) * src.token_stride + (is_q ? r0 + s0 : r0 + s0 - p.q_heads) * src.head_stride;
      if (r0 + s0 < r1) asm volatile("prefetch.global.L2 [%0];" ::"l"(x + e0));
    }
    __syncthreads();                                               // the last group's angles have been read
    for (int i = threadIdx.x; i < nt * p.half; i += QN_THREADS) {
      const int tt = i / p.half, j = i - tt * p.half;
      turn_of(p.positions[t0 + tt], p.inv_freq[j], p.factor, s_cos + tt * tpitch + j, s_sin + tt * tpitch + j);
    }
    __syncthreads();
    float cs[W], sn[W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const bool ok = mine && turns && live_token && i < angles;
      cs[i] = ok ? s_cos[t * tpitch + W * item + i] : 1.f;
      sn[i] = ok ? s_sin[t * tpitch + W * item + i] : 0.f;
    }

    // heads [h, end) of q or k, this slot's every per_token-th; whole warps go through together
    auto walk = [&](const gc_heads_t& src, const gc_heads_t& dst, const void* weight, int h, int end) {
      if (h >= end) return;
      const T* x = static_cast<const T*>(src.data) + (t0 + t) * src.token_stride + (h + s0) * src.head_stride;
      T* o = static_cast<T*>(dst.data) + (t0 + t) * dst.token_stride + (h + s0) * dst.head_stride;
      const int64_t xs = per_token * src.head_stride, os = per_token * dst.head_stride;
      auto load = [&](bool ok, uint4* a, uint4* b) {
        *a = *b = make_uint4(0, 0, 0, 0);
        if (ok) {
          *a = *reinterpret_cast<const uint4*>(x + e0);
          *b = *reinterpret_cast<const uint4*>(x + e1);
        }
      };
      bool ok = mine && live_token && h + s0 < end;
      uint4 a, b;
      load(ok, &a, &b);
      float w0[W], w1[W];
#pragma unroll
      for (int i = 0; i < W; ++i) w0[i] = w1[i] = 1.f;
      if (p.norm && weight && mine) {
        const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const T*>(weight) + e0), b = *reinterpret_cast<const uint4*>(static_cast<const T*>(weight) + e1);
#pragma unroll
        for (int i = 0; i < W; ++i) {
          w0[i] = to_f<T>(reinterpret_cast<const T*>(&a)[i]);
          w1[i] = to_f<T>(reinterpret_cast<const T*>(&b)[i]);
        }
      }
      for (; h < end; h += per_token) {
        float y0[W], y1[W];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
          y0[i] = to_f<T>(reinterpret_cast<const T*>(&a)[i]);
          y1[i] = to_f<T>(reinterpret_cast<const T*>(&b)[i]);
          sum = fmaf(y0[i], y0[i], fmaf(y1[i], y1[i], sum));
        }
        const bool next = mine && live_token && h + per_token + s0 < end;
        x += xs;
        load(next, &a, &b);
        if (mine && live_token && h + 2 * per_token + s0 < end) {       // and the one after it on its way to the L2
          asm volatile("prefetch.global.L2 [%0];" ::"l"(x + xs + e0));
          if (!INTERLEAVED) asm volatile("prefetch.global.L2 [%0];" ::"l"(x + xs + e1));
        }
        if (p.norm) {
          for (int d = L >> 1; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
          const float inv = rsqrtf(fmaf(sum, inv_d, p.eps));
#pragma unroll
          for (int i = 0; i < W; ++i) {
            y0[i] *= inv * w0[i];
            y1[i] *= inv * w1[i];
          }
        }
        if (turns && angles >= W) {                              // all pairs of the lane
#pragma unroll
          for (int i = 0; i < W; ++i) turn(y0, y1, i, cs[i], sn[i]);
        } else if (INTERLEAVED && angles > 0) {                  // the first few
#pragma unroll
          for (int i = 0; i < W; ++i)
            if (i < angles) turn(y0, y1, i, cs[i], sn[i]);
        }
        if (ok) {
          *reinterpret_cast<uint4*>(o + e0) = pack16<T>(y0);
          *reinterpret_cast<uint4*>(o + e1) = pack16<T>(y1);
        }
        o += os;
        ok = next;
      }
    };
    walk(p.q, p.q_out, p.q_weight, r0, min(r1, p.q_heads));
    walk(p.k, p.k_out, p.k_weight, max(r0 - p.q_heads, 0), r1 - p.q_heads);
  }
}

static bool aligned_heads(const gc_heads_t& h, int heads, int w, int esz) {
  return heads == 0 || (reinterpret_cast<uintptr_t>(h.data) % 16 == 0 && h.token_stride % w == 0 && h.head_stride % w == 0 && w * esz == 16);
}

template <typename K>
static cudaError_t launch_t(K kern, const QkParams& p, dim3 grid, size_t smem, cudaStream_t s) {
  if (smem > 48 * 1024) {
    cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), smem);
    if (e != cudaSuccess) return e;
  }
  return launch_following(kern, grid, QN_THREADS, smem, s, p);
}

cudaError_t launch_qk_norm_rope(const gc_qk_norm_rope_t& d, int num_sms, cudaStream_t s) {
  const bool f32 = d.dtype == GC_F32;
  const int esz = f32 ? 4 : 2;
  const int wv = 16 / esz;
  const bool vec = d.head_dim % wv == 0 && aligned_heads(d.q, d.q_heads, wv, esz) && aligned_heads(d.k, d.k_heads, wv, esz) &&
                   aligned_heads(d.q_out, d.q_heads, wv, esz) && aligned_heads(d.k_out, d.k_heads, wv, esz) &&
                   reinterpret_cast<uintptr_t>(d.q_weight) % 16 == 0 && reinterpret_cast<uintptr_t>(d.k_weight) % 16 == 0;
  // both halves of every pair in one lane's two vectors
  const bool pairs = vec && d.head_dim % (2 * wv) == 0 && (d.interleaved || ((d.rot_dim / 2) % wv == 0 && (d.head_dim - d.rot_dim) % (2 * wv) == 0));
  const int w = vec ? wv : 1;
  const int lanes = pairs ? d.head_dim / (2 * wv) : (d.head_dim + w - 1) / w;
  int log_l = 0;
  while (log_l < 5 && (1 << log_l) < lanes) ++log_l;
  const int slots = QN_THREADS >> log_l;
  QkParams p = {};
  p.q = d.q; p.k = d.k; p.q_out = d.q_out; p.k_out = d.k_out;
  p.q_weight = d.q_weight; p.k_weight = d.k_weight;
  p.positions = d.positions; p.inv_freq = d.inv_freq;
  p.tokens = d.tokens;
  p.q_heads = d.q_heads; p.rows = d.q_heads + d.k_heads;
  p.D = d.head_dim; p.half = d.rot_dim / 2; p.interleaved = d.interleaved; p.norm = d.norm;
  p.eps = d.eps; p.factor = d.attention_factor;
  p.log_l = log_l;
  // Four tokens per CTA keep its 256 threads busy while the angles are evaluated; with few tokens one per CTA, its heads
  // spread over as many CTAs as there are SMs (each evaluates the angles again: a few hundred clocks, all at once).
  p.tb = d.tokens >= 8LL * num_sms ? 4 : 1;
  int64_t parts = 1;
  if (d.tokens < num_sms) {
    parts = num_sms / d.tokens;
    const int most = (p.rows + slots - 1) / slots;
    if (parts > most) parts = most;
  }
  p.rows_per_cta = static_cast<int>((p.rows + parts - 1) / parts);
  const int64_t gx = (d.tokens + p.tb - 1) / p.tb;
  if (gx > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(gx), static_cast<unsigned>((p.rows + p.rows_per_cta - 1) / p.rows_per_cta));
  using bf16 = __nv_bfloat16;
  if (pairs) {
    // With many tokens four to a CTA, so that a thread's angles and weights serve several rows, and as many CTAs as fit at
    // once (three per SM), which walk over the groups; two to a CTA where four would leave SMs without work.  (A CTA has at least
    // eight rows at a time, so a token at least two.)
    dim3 pg = grid;
    if (d.tokens >= 4LL * num_sms) {
      p.tb = d.tokens >= 8LL * num_sms ? 4 : 2;
      const int64_t groups = (d.tokens + p.tb - 1) / p.tb;
      pg.x = static_cast<unsigned>(groups < 3LL * num_sms ? groups : 3LL * num_sms);
    }
    const size_t smem = 2 * static_cast<size_t>(p.tb) * ((p.half + wv - 1) / wv * wv) * 4;
    if (f32) return d.interleaved ? launch_t(qk_norm_rope_pairs_kernel<float, 4, true>, p, pg, smem, s) : launch_t(qk_norm_rope_pairs_kernel<float, 4, false>, p, pg, smem, s);
    return d.interleaved ? launch_t(qk_norm_rope_pairs_kernel<bf16, 8, true>, p, pg, smem, s) : launch_t(qk_norm_rope_pairs_kernel<bf16, 8, false>, p, pg, smem, s);
  }
  const size_t smem = (static_cast<size_t>(slots) * ((d.head_dim + 3) & ~3) + 2 * static_cast<size_t>(p.tb) * ((p.half + 3) & ~3)) * 4;
  if (f32) {
    if (!vec) return launch_t(qk_norm_rope_kernel<float, 1, 8>, p, grid, smem, s);
    return lanes > 32 ? launch_t(qk_norm_rope_kernel<float, 4, 2>, p, grid, smem, s) : launch_t(qk_norm_rope_kernel<float, 4, 1>, p, grid, smem, s);
  }
  return vec ? launch_t(qk_norm_rope_kernel<bf16, 8, 1>, p, grid, smem, s) : launch_t(qk_norm_rope_kernel<bf16, 1, 8>, p, grid, smem, s);
}

}  // namespace gc
