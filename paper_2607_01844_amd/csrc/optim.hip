// AdamW over many tensors and the gradients' sum of squares (gfx950).
//   g' = c g, c = max_norm / max(sqrt(sumsq), max_norm);
//   m' = b1 m + (1 - b1) g',  v' = b2 v + (1 - b2) g'^2;
//   w' = (1 - lr wd) w - lr / (1 - b1^t) m' / (sqrt(v') / sqrt(1 - b2^t) + eps).
// The tensors' addresses travel as kernel arguments, so a call uploads nothing and a
// captured one replays with the addresses it was given; a launch's workgroups are
// dealt out over the pieces of all its tensors, a piece each, neighbours on one XCD.
// Bound by the HBM stream: 28 bytes an element with fp32 states, weights and a bf16
// copy (619 M elements: 3.00 ms, 5.8 TB/s), 16 with 8-bit states (1.71 ms, 5.8 TB/s;
// a copy of 2 GiB moves 5.6 to 5.9).  Whole pieces take a path of their own: with
// every access behind its own test the 8-bit step took 1.95 ms.
//
// 8-bit states.  Blocks of 128 elements share a power of two u, 2^-14 (m) or 2^-30
// (v) of the one at or below their largest value; a value x is held as the exponent and
// the first three bits of mantissa of |x| + u, counted from u: segments of eight
// equal steps, each segment twice as wide as the one before (as telephony compands
// speech), the first ending at u.  What is cut off is rounded up or down at random
// with the right mean (at fp32's end, above 1.875 * 2^127, down): v moves by a few
// percent a step or less, which the nearest of steps of 1/8 would never follow.  A v above 0 is never held as 0, so that m / sqrt(v)
// stays bounded where v is small beside its block.  m', v' are formed in fp32 without
// contraction, so that codes are a function of the inputs alone.
#include <algorithm>

#include "common.h"

namespace moe {
namespace {

constexpr int MANY = 48;     // tensors of a launch (their table within the argument space)
// Groups of four elements a lane, 1024 apart: a workgroup's piece is 1024 of them.
// 619 M elements: 32-bit step 3.00 ms with one, 3.12 with two, 3.16 with four; 8-bit
// step 1.85, 1.71, 1.72; reading 8-bit states 1.06, 1.14, 1.14.
template <int BITS>
constexpr int GROUPS = BITS == 8 ? 2 : 1;
constexpr int GROUPS_READ = 1;
constexpr int SUM_PIECE = 16384;
constexpr int SUM_GRID = 2048;
constexpr int64_t MAX_GRID = int64_t{1} << 23;  // workgroups of a launch, 2^31 lanes

struct Tensors {
  moe_param p[MANY];
  int64_t first[MANY + 1];  // pieces before each
  int count;
};

// The tensor that piece c belongs to (uniform).
__device__ __forceinline__ int tensor_of(const Tensors& a, int64_t c) {
  int lo = 0, n = a.count;
  while (n > 1) {
    const int half = n >> 1;
    if (a.first[lo + half] <= c) {
      lo += half;
      n -= half;
    } else {
      n = half;
    }
  }
  return lo;
}

// A workgroup's first piece: those of one XCD (every eighth workgroup) are neighbours.
__device__ __forceinline__ int64_t first_piece() {
  const int64_t b = blockIdx.x, full = gridDim.x & ~7u;
  return b < full ? (b & 7) * (full >> 3) + (b >> 3) : b;
}

// Four elements from i on (in: how many there are), fp32 or bf16.
__device__ __forceinline__ void load4(const void* p, int type, int64_t i, int in, float* f) {
  f[0] = f[1] = f[2] = f[3] = 0.0f;
  if (type == MOE_F32) {
    const float* q = static_cast<const float*>(p) + i;
    if (in == 4) {
      const float4 v = load_stream(reinterpret_cast<const float4*>(q));
      f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    } else {
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (k < in) f[k] = q[k];
    }
  } else {
    const uint16_t* q = static_cast<const uint16_t*>(p) + i;
    if (in == 4) {
      const uint2 v = load_stream(reinterpret_cast<const uint2*>(q));
      f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
    } else {
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (k < in) f[k] = bf16_to_f32(q[k]);
    }
  }
}
__device__ __forceinline__ void store4(float* p, int64_t i, int in, const float* f) {
  if (in == 4) {
    store_stream(reinterpret_cast<float4*>(p + i), make_float4(f[0], f[1], f[2], f[3]));
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (k < in) p[i + k] = f[k];
  }
}
// lo, hi: two bf16 each
__device__ __forceinline__ void store4h(uint16_t* p, int64_t i, int in, uint32_t lo, uint32_t hi) {
  if (in == 4) {
    store_stream(reinterpret_cast<uint2*>(p + i), make_uint2(lo, hi));
  } else {
    if (in > 0) p[i] = static_cast<uint16_t>(lo);
    if (in > 1) p[i + 1] = static_cast<uint16_t>(lo >> 16);
    if (in > 2) p[i + 2] = static_cast<uint16_t>(hi);
  }
}
__device__ __forceinline__ uint32_t load4b(const uint8_t* p, int64_t i, int in) {
  if (in == 4) return load_stream(reinterpret_cast<const uint32_t*>(p + i));
  uint32_t v = 0;
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < in) v |= static_cast<uint32_t>(p[i + k]) << (8 * k);
  return v;
}
__device__ __forceinline__ void store4b(uint8_t* p, int64_t i, int in, uint32_t v) {
  if (in == 4) {
    store_stream(reinterpret_cast<uint32_t*>(p + i), v);
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (k < in) p[i + k] = static_cast<uint8_t>(v >> (8 * k));
  }
}

// ------------------------------------------------------------- 8-bit states
constexpr int M_SPAN = 14, V_SPAN = 30;  // octaves of u below the block's largest

__device__ __forceinline__ uint32_t mix(uint32_t x, uint32_t k) {
  x ^= x >> 16;
  x *= k;
  return x ^ (x >> 15);
}
__device__ __forceinline__ uint32_t max_over_block(uint32_t v) {
  auto f = [](float a, float b) {
    return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
  };
  return __float_as_uint(over_lanes<32>(__uint_as_float(v), f));
}
template <bool SIGNED>
__device__ __forceinline__ float decode(uint32_t code, uint32_t scale) {
  const float u = __uint_as_float(scale << 23);
  const uint32_t c = SIGNED ? code & 127u : code;
  const float mag = __uint_as_float((c << 20) + (scale << 23)) - u;
  return SIGNED && (code & 128u) ? -mag : mag;
}
// The exponent of u for a block whose largest magnitude has the bits `top` (of v', which
// is not below 0, with the sign bit a NaN may have); 255 (every value NaN) where it is
// not finite.
template <bool SIGNED>
__device__ __forceinline__ uint32_t scale_of(uint32_t top) {
  const int e = static_cast<int>(top >> 23);
  return e >= 255 ? 255u : static_cast<uint32_t>(max(e - (SIGNED ? M_SPAN : V_SPAN), 1));
}
// r: 16 random bits at place 4, and a half below them (bit 3).  Codes of a block with
// scale 255 are not used.
template <bool SIGNED>
__device__ __forceinline__ uint32_t encode(float x, uint32_t scale, uint32_t r) {
  const float u = __uint_as_float(scale << 23);
  const uint32_t c = ((__float_as_uint(fabsf(x) + u) + r) >> 20) - (scale << 3);
  if (SIGNED) return c | (__float_as_uint(x) >> 24 & 128u);
  return max(c, min(__float_as_uint(x), 1u));
}
// Four codes of a block with one of the last scales (the largest value in fp32's last
// octave, or not finite): at most the last code that stands for a finite value, else
// 1.875 * 2^127 and what lies above it could round up to the code of 2^128, an infinity.
// Other blocks' codes stay below by themselves, so none of them is compared: the scale is.
template <bool SIGNED>
__device__ __forceinline__ uint32_t last_codes(uint32_t codes, uint32_t scale) {
  if (scale == 255u) return 0u;
  const uint32_t most = 8u * (255u - scale) - 1u;
  uint32_t out = 0;
  for (int k = 0; k < 32; k += 8) {
    const uint32_t c = codes >> k & 255u, sign = SIGNED ? c & 128u : 0u;
    out |= (min(c - sign, most) | sign) << k;
  }
  return out;
}

// ------------------------------------------------------------------- AdamW
// The root within a unit in the last place; the instruction takes values below the
// normal numbers as 0, so small ones are scaled first.  With the reciprocal's unit
// the update is some 2^-22 of itself off, a tenth of a weight's own rounding where
// steps are a hundredth of weights (an IEEE root and division took 30 more
// instructions an element).
__device__ __forceinline__ float root_of(float v) {
  const bool small = v < 0x1p-96f;
  const float r = __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v);
  return small ? r * 0x1p-32f : r;
}

// A step's numbers, found in 64 bits and rounded once.
struct Step {
  float b1, a1, b2, a2, eps, keep, rate, root;  // a = 1 - b; root = 1 / sqrt(1 - b2^t)
};
__host__ __device__ inline double power(double b, uint32_t t) {
  double r = 1.0;
  for (; t; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}
__host__ __device__ inline Step step_numbers(double lr, double b1, double b2, double eps, double wd,
                                             uint32_t t) {
#pragma clang fp contract(off)  // the device's numbers are the host's
  Step s;
  s.b1 = static_cast<float>(b1);
  s.a1 = static_cast<float>(1.0 - b1);
  s.b2 = static_cast<float>(b2);
  s.a2 = static_cast<float>(1.0 - b2);
  s.eps = static_cast<float>(eps);
  s.keep = static_cast<float>(1.0 - lr * wd);
  s.rate = static_cast<float>(lr / (1.0 - power(b1, t)));
  s.root = static_cast<float>(1.0 / sqrt(1.0 - power(b2, t)));
  return s;
}

struct StepArgs {
  Step step;  // where lr and t are the host's
  double lr, b1, b2, eps, wd, max_norm;
  const float* lr_dev;
  const int32_t* step_dev;
  const float* sumsq;
  uint32_t t, seed, first_tensor;
};

// A piece's elements base + 1024 u .. + 3 of this lane.  WHOLE: the tensor holds all
// of the piece, and no access asks whether it may.
template <int BITS, bool WHOLE>
__device__ __forceinline__ void adamw_piece(const moe_param& p, int64_t base, const Step& st,
                                            float clip, uint32_t key) {
  constexpr int U = GROUPS<BITS>;
  float w[U][4], g[U][4], m[U][4], v[U][4];
  uint32_t mc[U], vc[U], ms[U], vs[U];
  int in[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = base + 1024 * u;
    in[u] = WHOLE ? 4 : static_cast<int>(min<int64_t>(max<int64_t>(p.n - i, 0), 4));
    load4(p.w, p.w_type, i, in[u], w[u]);
    load4(p.g, p.g_type, i, in[u], g[u]);
    if constexpr (BITS == 32) {
      load4(p.m, MOE_F32, i, in[u], m[u]);
      load4(p.v, MOE_F32, i, in[u], v[u]);
    } else {
      mc[u] = load4b(static_cast<const uint8_t*>(p.m), i, in[u]);
      vc[u] = load4b(static_cast<const uint8_t*>(p.v), i, in[u]);
      ms[u] = in[u] > 0 ? p.m_scale[i >> 7] : 0;
      vs[u] = in[u] > 0 ? p.v_scale[i >> 7] : 0;
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = base + 1024 * u;
    uint32_t r[4];
    uint32_t top_m = 0, top_v = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma clang fp contract(off)
      if constexpr (BITS == 8) {
        m[u][k] = decode<true>(mc[u] >> (8 * k) & 255u, ms[u]);
        v[u][k] = decode<false>(vc[u] >> (8 * k) & 255u, vs[u]);
      }
      const float x = g[u][k] * clip;
      m[u][k] = st.b1 * m[u][k] + st.a1 * x;
      v[u][k] = st.b2 * v[u][k] + st.a2 * (x * x);
      top_m = max(top_m, __float_as_uint(m[u][k]) & 0x7fffffffu);
      top_v = max(top_v, __float_as_uint(v[u][k]));
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      w[u][k] = st.keep * w[u][k] -
                st.rate * (m[u][k] * __builtin_amdgcn_rcpf(root_of(v[u][k]) * st.root + st.eps));
    if (BITS == 8 || p.w_type == MOE_BF16) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        r[k] = mix(static_cast<uint32_t>(i + k) * 0x9E3779B9u + key, 0x6A09E667u);
    }
    if constexpr (BITS == 32) {
      store4(static_cast<float*>(p.m), i, in[u], m[u]);
      store4(static_cast<float*>(p.v), i, in[u], v[u]);
    } else {
      const uint32_t sm = scale_of<true>(max_over_block(top_m));
      const uint32_t sv = scale_of<false>(max_over_block(top_v));
      uint32_t cm = 0, cv = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        cm |= encode<true>(m[u][k], sm, (r[k] << 4 & 0xffff0u) | 8u) << (8 * k);
        cv |= encode<false>(v[u][k], sv, (r[k] >> 12 & 0xffff0u) | 8u) << (8 * k);
      }
      if (sm >= 254u - M_SPAN) cm = last_codes<true>(cm, sm);
      if (sv >= 254u - V_SPAN) cv = last_codes<false>(cv, sv);
      store4b(static_cast<uint8_t*>(p.m), i, in[u], cm);
      store4b(static_cast<uint8_t*>(p.v), i, in[u], cv);
      if ((threadIdx.x & 31) == 0 && in[u] > 0) {
        p.m_scale[i >> 7] = static_cast<uint8_t>(sm);
        p.v_scale[i >> 7] = static_cast<uint8_t>(sv);
      }
    }
    if (p.w_type == MOE_F32) {
      store4(static_cast<float*>(p.w), i, in[u], w[u]);
      if (p.w_copy)
        store4h(p.w_copy, i, in[u], pack_bf16x2(w[u][0], w[u][1]), pack_bf16x2(w[u][2], w[u][3]));
    } else {
      // up or down at random with the right mean: a step is a small part of a
      // bf16 weight's last bit
      uint32_t b[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t x = __float_as_uint(w[u][k]);
        // (an infinity stays one; a NaN is left as it is, or it could wrap to a number)
        b[k] = w[u][k] != w[u][k] ? x | 0x400000u : x + (r[k] * 0xBB67AE85u >> 16);
      }
      store4h(static_cast<uint16_t*>(p.w), i, in[u], b[0] >> 16 | (b[1] & 0xffff0000u),
              b[2] >> 16 | (b[3] & 0xffff0000u));
    }
  }
}

template <int BITS>
__global__ __launch_bounds__(256) void adamw_kernel(const Tensors a, const StepArgs o) {
  constexpr int PIECE = 1024 * GROUPS<BITS>;
  __shared__ Step shared_step;
  __shared__ uint32_t shared_t;
  const int tid = threadIdx.x;
  float clip = 1.0f;
  if (o.sumsq) {
    const double q = *o.sumsq;
    // gradients that are not finite: the step is left out
    if (!(q >= 0.0 && q < __builtin_huge_val())) return;
    const double norm = sqrt(q);
    if (norm > o.max_norm) clip = static_cast<float>(o.max_norm / norm);
  }
  Step st = o.step;
  uint32_t t = o.t;
  if (o.lr_dev || o.step_dev) {
    if (tid == 0) {
      if (o.step_dev) t = static_cast<uint32_t>(max(*o.step_dev, 1));
      shared_step = step_numbers(o.lr_dev ? static_cast<double>(*o.lr_dev) : o.lr, o.b1, o.b2,
                                 o.eps, o.wd, t);
      shared_t = t;
    }
    __syncthreads();
    st = shared_step;
    t = shared_t;
  }
  for (int64_t c = first_piece(); c < a.first[a.count]; c += gridDim.x) {
    const int j = tensor_of(a, c);
    const moe_param& p = a.p[j];
    const int64_t start = (c - a.first[j]) * PIECE;
    uint32_t key = 0;
    if (BITS == 8 || p.w_type == MOE_BF16) {
      key = o.seed + t * 0x85A308D3u + (o.first_tensor + j) * 0x9E3779B9u;
      key = mix(mix(key, 0x6A09E667u), 0xBB67AE85u);
    }
    if (p.n - start >= PIECE)
      adamw_piece<BITS, true>(p, start + 4 * tid, st, clip, key);
    else
      adamw_piece<BITS, false>(p, start + 4 * tid, st, clip, key);
  }
}

// The values that 8-bit states stand for, into w (those of m) and w_copy (of v), which
// a launch's table has no other use for.
template <bool WHOLE>
__device__ __forceinline__ void states_piece(const moe_param& p, int64_t base) {
  constexpr int U = GROUPS_READ;
  uint32_t mc[U], vc[U], ms[U], vs[U];
  int in[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = base + 1024 * u;
    in[u] = WHOLE ? 4 : static_cast<int>(min<int64_t>(max<int64_t>(p.n - i, 0), 4));
    mc[u] = load4b(static_cast<const uint8_t*>(p.m), i, in[u]);
    vc[u] = load4b(static_cast<const uint8_t*>(p.v), i, in[u]);
    ms[u] = in[u] > 0 ? p.m_scale[i >> 7] : 0;
    vs[u] = in[u] > 0 ? p.v_scale[i >> 7] : 0;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = base + 1024 * u;
    float m[4], v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[k] = decode<true>(mc[u] >> (8 * k) & 255u, ms[u]);
      v[k] = decode<false>(vc[u] >> (8 * k) & 255u, vs[u]);
    }
    store4(static_cast<float*>(p.w), i, in[u], m);
    store4(reinterpret_cast<float*>(p.w_copy), i, in[u], v);
  }
}
__global__ __launch_bounds__(256) void adamw_states_kernel(const Tensors a) {
  constexpr int PIECE = 1024 * GROUPS_READ;
  for (int64_t c = first_piece(); c < a.first[a.count]; c += gridDim.x) {
    const int j = tensor_of(a, c);
    const moe_param& p = a.p[j];
    const int64_t start = (c - a.first[j]) * PIECE;
    if (p.n - start >= PIECE)
      states_piece<true>(p, start + 4 * threadIdx.x);
    else
      states_piece<false>(p, start + 4 * threadIdx.x);
  }
}

// ---------------------------------------------------------- sum of squares
__device__ __forceinline__ float squares32(const uint4& v) {
  const float a = __uint_as_float(v.x), b = __uint_as_float(v.y), c = __uint_as_float(v.z),
              d = __uint_as_float(v.w);
  return (a * a + b * b) + (c * c + d * d);
}
__device__ __forceinline__ float squares16(const uint4& v) {
  const uint32_t b[4] = {v.x, v.y, v.z, v.w};
  float f = 0.0f;
#pragma unroll
  for (int k = 0; k < 4; ++k) f += bf16_lo(b[k]) * bf16_lo(b[k]) + bf16_hi(b[k]) * bf16_hi(b[k]);
  return f;
}

// part[workgroup]: fp32 within a lane's share of a piece, 64 bits beyond.
__global__ __launch_bounds__(256) void grad_sumsq_kernel(const Tensors a, double* __restrict__ part) {
  __shared__ double sums[4];
  double s = 0.0;
  // a workgroup's pieces are neighbours: HBM gives such reads 7 TB/s, pieces dealt out
  // in turn 5.8 (1.24 GB: 184 us, 6.7 TB/s)
  const int64_t per = (a.first[a.count] + gridDim.x - 1) / gridDim.x;
  const int64_t last = min<int64_t>(a.first[a.count], (blockIdx.x + 1) * per);
  for (int64_t c = blockIdx.x * per; c < last; ++c) {
    const int j = tensor_of(a, c);
    const moe_param& p = a.p[j];
    const int64_t base = (c - a.first[j]) * SUM_PIECE;
    float f = 0.0f;
    const int64_t end = min<int64_t>(p.n, base + SUM_PIECE);
    if (end - base == SUM_PIECE) {
      // a whole piece: eight loads of 16 bytes a lane in flight
      const uint4* q = reinterpret_cast<const uint4*>(
          static_cast<const char*>(p.g) + base * (p.g_type == MOE_F32 ? 4 : 2));
      const int batches = p.g_type == MOE_F32 ? 2 : 1;
      for (int k = 0; k < batches; ++k) {
        uint4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = load_stream(q + (k * 8 + u) * 256 + threadIdx.x);
#pragma unroll
        for (int u = 0; u < 8; ++u) f += p.g_type == MOE_F32 ? squares32(v[u]) : squares16(v[u]);
      }
    } else if (p.g_type == MOE_F32) {
      const float* q = static_cast<const float*>(p.g);
      for (int64_t i = base + threadIdx.x; i < end; i += 256) f += q[i] * q[i];
    } else {
      const uint16_t* q = static_cast<const uint16_t*>(p.g);
      for (int64_t i = base + 8 * threadIdx.x; i < end; i += 2048) {
        if (end - i >= 8)
          f += squares16(load_stream(reinterpret_cast<const uint4*>(q + i)));
        else
          for (int64_t k = i; k < end; ++k) f += bf16_to_f32(q[k]) * bf16_to_f32(q[k]);
      }
    }
    s += f;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}
__global__ __launch_bounds__(1024) void grad_sumsq_join_kernel(const double* __restrict__ part,
                                                               int64_t n, float* __restrict__ out) {
  __shared__ double sums[16];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += part[i];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int w = 0; w < 16; ++w) s += sums[w];
    *out = static_cast<float>(s);
  }
}

// f(tensors of one launch, index of the first) over a list, MANY at a time;
// tensors without elements are left out (false: there was no other).
template <typename F>
bool in_launches(const moe_param* params, int count, int64_t piece, F&& f) {
  Tensors a;
  int index[MANY];
  bool any = false;
  a.count = 0;
  a.first[0] = 0;
  for (int i = 0; i < count; ++i) {
    if (params[i].n > 0) {
      // a tensor's number is its place in the list: no gap within a launch
      if (a.count > 0 && index[a.count - 1] != i - 1) {
        f(a, index[0]);
        a.count = 0;
      }
      any = true;
      a.p[a.count] = params[i];
      index[a.count] = i;
      a.first[a.count + 1] = a.first[a.count] + ceil_div(params[i].n, piece);
      ++a.count;
    }
    if (a.count > 0 && (a.count == MANY || i + 1 == count)) {
      f(a, index[0]);
      a.count = 0;
    }
  }
  return any;
}

}  // namespace

hipError_t launch_adamw(const moe_param* params, int count, int bits, const moe_adamw_options& opt,
                        hipStream_t s) {
  StepArgs o;
  o.t = static_cast<uint32_t>(opt.step_device ? 1 : opt.step);
  o.step = step_numbers(opt.lr, opt.beta1, opt.beta2, opt.eps, opt.weight_decay, o.t);
  o.lr = opt.lr; o.b1 = opt.beta1; o.b2 = opt.beta2; o.eps = opt.eps; o.wd = opt.weight_decay;
  o.max_norm = opt.max_norm;
  o.lr_dev = opt.lr_device; o.step_dev = opt.step_device; o.sumsq = opt.grad_sumsq;
  o.seed = opt.seed;
  prof_begin(K_ADAMW, s);
  const bool any = in_launches(params, count, 1024 * (bits == 32 ? GROUPS<32> : GROUPS<8>), [&](const Tensors& a, int first) {
    o.first_tensor = static_cast<uint32_t>(first);
    const unsigned grid = static_cast<unsigned>(std::min(a.first[a.count], MAX_GRID));
    if (bits == 32)
      adamw_kernel<32><<<grid, 256, 0, s>>>(a, o);
    else
      adamw_kernel<8><<<grid, 256, 0, s>>>(a, o);
  });
  prof_end(K_ADAMW, s);
  return any ? hipGetLastError() : hipSuccess;
}

hipError_t launch_adamw_states(const moe_param* params, int count, float* const* m, float* const* v,
                               hipStream_t s) {
  prof_begin(K_ADAMW_STATES, s);
  const bool any = in_launches(params, count, 1024 * GROUPS_READ, [&](Tensors& a, int first) {
    for (int j = 0; j < a.count; ++j) {
      a.p[j].w = m[first + j];
      a.p[j].w_copy = reinterpret_cast<uint16_t*>(v[first + j]);
    }
    const unsigned grid = static_cast<unsigned>(std::min(a.first[a.count], MAX_GRID));
    adamw_states_kernel<<<grid, 256, 0, s>>>(a);
  });
  prof_end(K_ADAMW_STATES, s);
  return any ? hipGetLastError() : hipSuccess;
}

// Partial sums of all launches of a list.
static int64_t sumsq_parts(const moe_param* params, int count) {
  int64_t n = 0;
  in_launches(params, count, SUM_PIECE, [&](const Tensors& a, int) {
    n += std::min<int64_t>(a.first[a.count], SUM_GRID);
  });
  return n;
}
size_t grad_sumsq_ws_bytes(const moe_param* params, int count) {
  return align_up(sizeof(double) * static_cast<size_t>(std::max<int64_t>(1, sumsq_parts(params, count))), 256);
}

hipError_t launch_grad_sumsq(const moe_param* params, int count, float* sumsq, void* ws,
                             hipStream_t s) {
  double* part = static_cast<double*>(ws);
  int64_t n = 0;
  prof_begin(K_GRAD_SUMSQ, s);
  in_launches(params, count, SUM_PIECE, [&](const Tensors& a, int) {
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(a.first[a.count], SUM_GRID));
    grad_sumsq_kernel<<<grid, 256, 0, s>>>(a, part + n);
    n += grid;
  });
  grad_sumsq_join_kernel<<<1, 1024, 0, s>>>(part, n, sumsq);
  prof_end(K_GRAD_SUMSQ, s);
  return hipGetLastError();
}

}  // namespace moe
