// MXFP4: quantisation of bf16 matrices to 4-bit values with one power-of-two
// scale per 32, back to the values they stand for, and the expert layer's
// forward on them (the products are in mxfp4_gemm.h).
//
// A block of 32 consecutive k has the scale 2^(floor(log2 max|v|) - 2), kept in
// [2^-127, 2^127] (so the largest value lands in [4, 8) and saturates at 6), and
// each value is v / scale rounded to the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6,
// ties to the even code, by the hardware's scaled conversion (checked against
// that rule over all bf16 values at scales from 2^-127 to 2^127).  A block with
// a NaN or an infinity has the scale byte 255, and stands for NaN.
// The quantisers read each value once, 16 bytes (along rows) or 4 (along
// columns) a lane, and are bound by that stream: 64 matrices of 2048 x 1408 (369 MB)
// along columns 92 to 129 us with 98 MB written, back to bf16 92 to 105, where a copy
// of the same bytes takes 94; 1100 x 520 along rows 3.1 and 4.3 us, launches.
// (Twice the bytes a lane along columns is no faster.)
// Products and silu are fp32; the activations are rounded to MXFP4, the down
// product's operand, and each expert row of the result to bf16 before moe_combine
// weighs the rows in fp32, as in the bf16 layer: half the bytes that fp32 rows
// would write and read again (y against 64 bits: 0.0024 of its norm off, 0.0017
// with one rounding at the end).
#include <algorithm>

#include "mxfp4_gemm.h"

namespace moe {
using namespace gemm;
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <int SEL>
__device__ __forceinline__ uint32_t fp4_pair_bf16(uint32_t old, uint32_t two, float scale) {
  return static_cast<uint32_t>(
      __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2, two), scale, SEL));
}
// The largest bf16 magnitude of a packed pair, as fp32 bits of its magnitude.
__device__ __forceinline__ uint32_t pair_top(uint32_t v) {
  return max((v << 16) & 0x7fffffffu, v & 0x7fff0000u);
}

// Quantised rows on their way into a layer: each token's scales go to its
// permuted rows, whose token is noted (dst: see moe_permute), and the last
// workgroup forms the table of row tiles of the products that follow.
struct Scatter {
  const int32_t* dst;      // [T][k]; null: scales stay in row order
  const int32_t* offsets;  // [E_loc + 1]
  int32_t *tok, *mt;       // [cap], [E_loc + 1]
  int64_t cap;
  int k, E_loc, tile;      // tile: rows of a row tile
};

// mt[e] = row tiles of the experts before e (256 threads, up to 1024 experts).
__device__ __forceinline__ void tile_table(const Scatter& c) {
  __shared__ int wsum[4];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int v[4], sum = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = 4 * threadIdx.x + i;
    v[i] = e < c.E_loc ? (c.offsets[e + 1] - c.offsets[e] + c.tile - 1) / c.tile : 0;
    sum += v[i];
  }
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(incl, o, 64);
    if (lane >= o) incl += u;
  }
  if (lane == 63) wsum[w] = incl;
  __syncthreads();
  int at = incl - sum;
  for (int q = 0; q < w; ++q) at += wsum[q];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = 4 * threadIdx.x + i;
    if (e < c.E_loc) c.mt[e] = at;
    at += v[i];
    if (e == c.E_loc - 1) c.mt[c.E_loc] = at;
  }
}

// Along rows: q [rows][kq], s [ceil(K / 256)][rows][8] of src [rows][K] (batches
// of `rows` rows follow one another).  Four lanes a block, 8 values each, 32 the
// eight blocks whose scales lie together; W lanes along K, the rest of the
// workgroup along rows.  SCATTER: the scales go to s [ceil(K / 256)][cap][8].
template <int W, bool SCATTER>
__global__ __launch_bounds__(256) void mx_quant_kernel(const uint16_t* __restrict__ src, int64_t total,
                                                       int64_t rows, int K, uint8_t* __restrict__ q,
                                                       uint8_t* __restrict__ s, Scatter sc) {
  constexpr int RPB = 256 / W;
  if constexpr (SCATTER) {
    if (blockIdx.x == gridDim.x - 1) {
      if (blockIdx.y == 0) tile_table(sc);
      return;
    }
  }
  const int nb = (K + 31) / 32, nkg = (nb + 7) / 8;
  const int u = blockIdx.y * W + threadIdx.x % W;  // 8 values of the row
  const int b = u >> 2, part = u & 3;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * RPB + threadIdx.x / W;
  if (r >= total || b >= 8 * nkg) return;  // whole groups of 32 lanes
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
  if (8 * u < K) v = *reinterpret_cast<const uint4*>(src + r * K + 8 * u);
  uint32_t top = max(max(pair_top(v.x), pair_top(v.y)), max(pair_top(v.z), pair_top(v.w)));
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1, 64)));
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2, 64)));
  const uint32_t e8 = mx_scale(top);
  const float scale = __uint_as_float(e8 << 23);
  uint32_t o = 0;
  o = fp4_pair_bf16<0>(o, v.x, scale);
  o = fp4_pair_bf16<1>(o, v.y, scale);
  o = fp4_pair_bf16<2>(o, v.z, scale);
  o = fp4_pair_bf16<3>(o, v.w, scale);
  if (b < nb) *reinterpret_cast<uint32_t*>(q + (r * nb + b) * 16 + 4 * part) = o;
  // the four even (odd) blocks' bytes in every lane of an even (odd) block
  uint32_t bytes = b < nb ? e8 << (8 * ((b & 7) >> 1)) : 0u;
  bytes |= static_cast<uint32_t>(__shfl_xor(static_cast<int>(bytes), 8, 64));
  bytes |= static_cast<uint32_t>(__shfl_xor(static_cast<int>(bytes), 16, 64));
  const int slot = part + 4 * ((b >> 1) & 3), odd = b & 1;  // 16 lanes of each parity
  const int64_t kg = b >> 3;
  if constexpr (SCATTER) {
    if (slot < sc.k) {
      const int64_t p = sc.dst[r * sc.k + slot];
      if (p >= 0) {
        *reinterpret_cast<uint32_t*>(s + (kg * sc.cap + p) * 8 + 4 * odd) = bytes;
        if (kg == 0 && odd == 0) sc.tok[p] = static_cast<int32_t>(r);
      }
    }
  } else if (slot == 0) {
    const int64_t batch = r / rows, rr = r - batch * rows;
    *reinterpret_cast<uint32_t*>(s + ((batch * nkg + kg) * rows + rr) * 8 + 4 * odd) = bytes;
  }
}

// Along columns: src [B][K][C] -> q [B][C][kq], s [B][ceil(K / 256)][C][8]: a
// workgroup takes 256 k of TC columns, a wave 32 of them (one block a column), a
// lane TC / 64 columns; values and scales leave through LDS, a column's 128 bytes
// together.
constexpr int TC = 128;
__global__ __launch_bounds__(512) void mx_quant_t_kernel(const uint16_t* __restrict__ src, int K, int C,
                                                         uint8_t* __restrict__ q,
                                                         uint8_t* __restrict__ s) {
  __shared__ __align__(16) uint4 vb[TC][8];  // 16-byte piece w of column c at w ^ (c / 2 % 8)
  __shared__ __align__(8) uint8_t sb[TC][8];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int nb = (K + 31) / 32, nkg = (nb + 7) / 8;
  const int c0 = blockIdx.x * TC, c = c0 + 2 * lane;
  const int kg = blockIdx.y, b = kg * 8 + w, k0 = 32 * b;
  const int64_t batch = blockIdx.z;
  const uint16_t* in = src + (batch * K + k0) * C + c;
  uint32_t v[32];
  if (k0 + 32 <= K && c < C) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = *reinterpret_cast<const uint32_t*>(in + static_cast<int64_t>(i) * C);
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      v[i] = c < C && k0 + i < K ? *reinterpret_cast<const uint32_t*>(in + static_cast<int64_t>(i) * C) : 0u;
  }
  uint32_t t0 = 0, t1 = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    t0 = max(t0, (v[i] << 16) & 0x7fffffffu);
    t1 = max(t1, v[i] & 0x7fff0000u);
  }
  const uint32_t e[2] = {mx_scale(t0), mx_scale(t1)};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float sc = __uint_as_float(e[h] << 23);
    uint32_t o[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = v[8 * p + 2 * i], hi = v[8 * p + 2 * i + 1];
        x[i] = h == 0 ? (lo & 0xffffu) | (hi << 16) : (lo >> 16) | (hi & 0xffff0000u);
      }
      uint32_t r = 0;
      r = fp4_pair_bf16<0>(r, x[0], sc);
      r = fp4_pair_bf16<1>(r, x[1], sc);
      r = fp4_pair_bf16<2>(r, x[2], sc);
      r = fp4_pair_bf16<3>(r, x[3], sc);
      o[p] = r;
    }
    vb[2 * lane + h][w ^ (lane & 7)] = make_uint4(o[0], o[1], o[2], o[3]);
    sb[2 * lane + h][mx_pos(w)] = b < nb ? static_cast<uint8_t>(e[h]) : 0;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < TC / 64; ++i) {
    const int cc = 64 * i + (threadIdx.x >> 3), piece = threadIdx.x & 7;
    if (c0 + cc < C && kg * 8 + piece < nb)
      *reinterpret_cast<uint4*>(q + ((batch * C + c0 + cc) * nb + kg * 8 + piece) * 16) =
          vb[cc][piece ^ ((cc >> 1) & 7)];
  }
  const int cc = threadIdx.x;
  if (cc < TC && c0 + cc < C)
    *reinterpret_cast<uint2*>(s + ((batch * nkg + kg) * C + c0 + cc) * 8) = *reinterpret_cast<const uint2*>(sb[cc]);
}

// dst [rows][K] bf16 of q, s (batches of `rows` rows): 8 values a thread of DR
// rows.  Every value is a bf16 (two significant bits, at least 2^-128).
constexpr int DR = 4;
template <int W>
__global__ __launch_bounds__(256) void mx_dequant_kernel(const uint8_t* __restrict__ q,
                                                         const uint8_t* __restrict__ s, int64_t total,
                                                         int64_t rows, int K, uint16_t* __restrict__ dst) {
  constexpr int RPB = 256 / W;
  const int nb = (K + 31) / 32, nkg = (nb + 7) / 8;
  const int u = blockIdx.y * W + threadIdx.x % W;
  const int b = u >> 2;
  if (8 * u >= K) return;
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * (RPB * DR) + threadIdx.x / W;
  uint32_t e8[DR], v[DR];
#pragma unroll
  for (int i = 0; i < DR; ++i) {
    const int64_t r = r0 + i * RPB < total ? r0 + i * RPB : total - 1;
    const int64_t batch = r / rows, rr = r - batch * rows;
    e8[i] = s[((batch * nkg + (b >> 3)) * rows + rr) * 8 + mx_pos(b)];
    v[i] = *reinterpret_cast<const uint32_t*>(q + (r * nb + b) * 16 + 4 * (u & 3));
  }
#pragma unroll
  for (int i = 0; i < DR; ++i) {
    const int64_t r = r0 + i * RPB;
    if (r >= total) return;
    uint32_t o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t c = v[i] >> (8 * j + 4 * h), m = c & 7u;
        // 0, 1/2 and (1 + m0 / 2) 2^(m / 2 - 1)
        const float a = m < 2 ? 0.5f * static_cast<float>(m)
                              : __uint_as_float(((126u + (m >> 1)) << 23) | ((m & 1u) << 22));
        x[h] = __builtin_ldexpf(c & 8u ? -a : a, static_cast<int>(e8[i]) - 127);
      }
      o[j] = e8[i] == 255u ? 0x7fc07fc0u : pack_bf16x2(x[0], x[1]);
    }
    *reinterpret_cast<uint4*>(dst + r * K + 8 * u) = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// Scales of the permuted rows, and each row's token: s_perm [nkg][cap][8].
__global__ __launch_bounds__(256) void mx_gather_scales_kernel(const uint8_t* __restrict__ s, int64_t T,
                                                               const int32_t* __restrict__ row_src, int k,
                                                               const int32_t* __restrict__ offsets,
                                                               int E_loc, int64_t cap,
                                                               uint8_t* __restrict__ s_perm,
                                                               int32_t* __restrict__ tok) {
  const int64_t p = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t M = offsets[E_loc];
  if (p >= M || p >= cap) return;
  int64_t t = row_src[p] / k;
  t = t < 0 ? 0 : t < T ? t : T - 1;
  const int64_t kg = blockIdx.y;
  *reinterpret_cast<uint2*>(s_perm + (kg * cap + p) * 8) =
      *reinterpret_cast<const uint2*>(s + (kg * T + t) * 8);
  if (kg == 0) tok[p] = static_cast<int32_t>(t);
}

int64_t kgroups(int64_t K) { return ceil_div(K, 256); }
int64_t kq_of(int64_t K) { return 16 * ceil_div(K, 32); }

struct FfnWs {
  int32_t *mt, *wk, *nz;
  uint8_t *act_q, *act_s, *s_perm;
  int32_t* tok;
  size_t bytes;
};
FfnWs carve_ffn(void* ws, int64_t cap, int E_loc, int d, int f, bool indirect) {
  char* p = static_cast<char*>(ws);
  size_t used = 0;
  auto take = [&](size_t n) {
    char* q = p + used;
    used += align_up(n, 256);
    return q;
  };
  const size_t c = static_cast<size_t>(cap);
  FfnWs w{};
  w.mt = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * (E_loc + 1)));
  w.wk = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * (E_loc + 1)));
  w.nz = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * (E_loc + 1)));
  w.act_q = reinterpret_cast<uint8_t*>(take(c * kq_of(f)));
  w.act_s = reinterpret_cast<uint8_t*>(take(c * 8 * kgroups(f)));
  if (indirect) {
    w.s_perm = reinterpret_cast<uint8_t*>(take(c * 8 * kgroups(d)));
    w.tok = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * c));
  }
  w.bytes = used;
  return w;
}

template <int MODE>
hipError_t run_mx(const MxArgs& a, bool small, int kid, hipStream_t s) {
  const int64_t g = std::max<int64_t>(1, device_cus() / NXCD) * NXCD;
  prof_begin(kid, s);
  if (small)
    mxfp4_gemm_kernel<MODE, TILE_S><<<static_cast<unsigned>(2 * g), MxGeom<TILE_S>::NTHR, 0, s>>>(a);
  else
    mxfp4_gemm_kernel<MODE, TILE><<<static_cast<unsigned>(g), MxGeom<TILE>::NTHR, 0, s>>>(a);
  prof_end(kid, s);
  return hipGetLastError();
}

}  // namespace

namespace {
// scatter: the layer's rows (see Scatter), one workgroup more
hipError_t quantize_rows(const uint16_t* src, int64_t B, int64_t R, int64_t C, uint8_t* q, uint8_t* s,
                         const Scatter* sc, hipStream_t st) {
  const int64_t units = 32 * kgroups(C);  // of 8 values, the last scales' padding included
  auto go = [&](auto W, auto SC) {
    mx_quant_kernel<W, SC><<<dim3(static_cast<unsigned>(ceil_div(B * R, 256 / W) + (SC ? 1 : 0)),
                                  static_cast<unsigned>(ceil_div(units, W))),
                             256, 0, st>>>(src, B * R, R, static_cast<int>(C), q, s, SC ? *sc : Scatter{});
  };
  // two rows a workgroup would pass the 2^32 threads of a launch from 2^25 - 1 rows on
  const bool many = B * R > int64_t{1} << 24;
  auto width = [&](auto SC) {
    if (units <= 32) go(std::integral_constant<int, 32>{}, SC);
    else if (units <= 64 || many) go(std::integral_constant<int, 64>{}, SC);
    else go(std::integral_constant<int, 128>{}, SC);
  };
  if (sc != nullptr) width(std::true_type{});
  else width(std::false_type{});
  return hipGetLastError();
}
}  // namespace

hipError_t launch_mx_quantize(const uint16_t* src, int64_t B, int64_t R, int64_t C, int transpose,
                              uint8_t* q, uint8_t* s, hipStream_t st) {
  if (B * R * C == 0) return hipSuccess;
  prof_begin(K_MX_QUANT, st);
  hipError_t e;
  if (transpose) {
    mx_quant_t_kernel<<<dim3(static_cast<unsigned>(ceil_div(C, 128)), static_cast<unsigned>(kgroups(R)),
                             static_cast<unsigned>(B)),
                        512, 0, st>>>(src, static_cast<int>(R), static_cast<int>(C), q, s);
    e = hipGetLastError();
  } else {
    e = quantize_rows(src, B, R, C, q, s, nullptr, st);
  }
  prof_end(K_MX_QUANT, st);
  return e;
}

hipError_t launch_mx_dequantize(const uint8_t* q, const uint8_t* s, int64_t B, int64_t rows, int64_t K,
                                uint16_t* dst, hipStream_t st) {
  if (B * rows * K == 0) return hipSuccess;
  prof_begin(K_MX_QUANT, st);
  const int64_t units = ceil_div(K, 8);
  auto go = [&](auto W) {
    mx_dequant_kernel<W><<<dim3(static_cast<unsigned>(ceil_div(B * rows, 256 / W * DR)),
                                static_cast<unsigned>(ceil_div(units, W))),
                           256, 0, st>>>(q, s, B * rows, rows, static_cast<int>(K), dst);
  };
  if (units <= 32) go(std::integral_constant<int, 32>{});
  else if (units <= 64) go(std::integral_constant<int, 64>{});
  else go(std::integral_constant<int, 128>{});
  prof_end(K_MX_QUANT, st);
  return hipGetLastError();
}

size_t mx_ffn_ws_bytes(int64_t cap, int E_loc, int d, int f, bool indirect) {
  return carve_ffn(nullptr, cap, E_loc, d, f, indirect).bytes;
}

namespace {
// The 128-row tile for experts of up to 128 rows on average, which fill one of
// them (64 experts of 16 rows, d = 2048, f = 1408, both products: 64 us against
// 69 on 256-row tiles; 128 rows 89 against 91; beyond the line 160 rows 117
// against 97, 128 experts of 512 rows, d = 4096, f = 1536 884 against 705), and
// where 256-row tiles would use less than two thirds of the CUs (12 experts of
// 256 rows, d = 520, f = 328: 21 us against 30; 16 of 512, d = 1024, f = 512 27
// against 33; beyond the line 16 of 1000 40 against 36).
bool small_tile(int64_t rows, int E_loc, int d, int f) {
  if (rows <= 128 * int64_t{E_loc}) return true;
  const int64_t cus = device_cus();
  const int64_t tiles = (std::min<int64_t>(rows, E_loc) + rows / TILE) *
                        std::max(ceil_div(f, TILE / 2), ceil_div(d, TILE));
  return 3 * tiles < 2 * cus * ceil_div(tiles, cus);
}

// The two products.  xs: the scales of the permuted rows ([..][s_rows][8]);
// tok: their rows of xq (null: the same); w.mt: the table of row tiles.
hipError_t products(const uint8_t* xq, int64_t x_rows, const uint8_t* xs, int64_t s_rows, const int32_t* tok,
                    const FfnWs& w, bool small, const int32_t* offsets, int E_loc, int64_t cap, int d,
                    int f, const uint8_t* const wq[3], const uint8_t* const wsc[3], uint16_t* y,
                    hipStream_t s) {
  const int S = small ? TILE_S : TILE;
  MxArgs a{};
  a.a = {xq, xs};
  a.a_tok = tok;
  a.a_rows = s_rows;
  a.a_bytes = x_rows * kq_of(d);
  a.b0 = {wq[0], wsc[0]};
  a.b1 = {wq[1], wsc[1]};
  a.act_q = w.act_q; a.act_s = w.act_s; a.cap = cap; a.y = y;
  a.t.offsets = offsets; a.t.mt_start = w.mt;
  a.t.E_loc = E_loc; a.t.d = d; a.t.f = f;
  a.t.NT = static_cast<int>(ceil_div(f, S / 2));
  if (hipError_t e = run_mx<MX_GATE_UP>(a, small, K_MX_GATE_UP, s); e != hipSuccess) return e;
  a.a = {w.act_q, w.act_s};
  a.a_tok = nullptr;
  a.a_rows = cap;
  a.a_bytes = cap * kq_of(f);
  a.b0 = {wq[2], wsc[2]};
  a.t.NT = static_cast<int>(ceil_div(d, S));
  return run_mx<MX_DOWN>(a, small, K_MX_DOWN, s);
}
}  // namespace

hipError_t launch_mx_ffn(const uint8_t* xq, const uint8_t* xs, int64_t x_rows, const int32_t* row_src,
                         int k, const int32_t* offsets, int E_loc, int64_t cap, int d, int f,
                         const uint8_t* const wq[3], const uint8_t* const wsc[3], uint16_t* y,
                         void* ws, hipStream_t s) {
  if (cap == 0) return hipSuccess;
  const bool indirect = row_src != nullptr;
  const FfnWs w = carve_ffn(ws, cap, E_loc, d, f, indirect);
  if (indirect) {
    prof_begin(K_MX_QUANT, s);
    mx_gather_scales_kernel<<<dim3(static_cast<unsigned>(ceil_div(cap, 256)),
                                   static_cast<unsigned>(kgroups(d))),
                              256, 0, s>>>(xs, x_rows, row_src, k, offsets, E_loc, cap, w.s_perm, w.tok);
    prof_end(K_MX_QUANT, s);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  const bool small = small_tile(cap, E_loc, d, f);  // the host knows the capacity alone
  if (hipError_t e = launch_gemm_sched(offsets, E_loc, small ? TILE_S : TILE, BK, w.mt, w.wk, w.nz, s);
      e != hipSuccess)
    return e;
  return products(xq, x_rows, indirect ? w.s_perm : xs, indirect ? cap : x_rows, indirect ? w.tok : nullptr,
                  w, small, offsets, E_loc, cap, d, f, wq, wsc, y, s);
}

namespace {
struct LayerWs {
  int32_t *offsets, *row_src, *dst;
  void *perm, *ffn;
  uint8_t* xq;
  uint16_t* y_perm;
  size_t bytes;
};
LayerWs carve_layer(void* ws, int64_t T, int E, int k, int E_loc, int d, int f) {
  const int64_t cap = T * std::min(k, E_loc);
  char* p = static_cast<char*>(ws);
  size_t used = 0;
  auto take = [&](size_t n) {
    char* q = p + used;
    used += align_up(n, 256);
    return q;
  };
  LayerWs w{};
  w.offsets = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * (E_loc + 1)));
  w.row_src = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * static_cast<size_t>(cap)));
  w.dst = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * static_cast<size_t>(T) * k));
  w.perm = take(permute_ws_bytes(T, E, k, E_loc));
  w.xq = reinterpret_cast<uint8_t*>(take(static_cast<size_t>(T) * kq_of(d)));
  w.y_perm = reinterpret_cast<uint16_t*>(take(sizeof(uint16_t) * static_cast<size_t>(cap) * d));
  w.ffn = take(mx_ffn_ws_bytes(cap, E_loc, d, f, true));
  w.bytes = used;
  return w;
}
}  // namespace

size_t mx_layer_ws_bytes(int64_t T, int E, int k, int E_loc, int d, int f) {
  return carve_layer(nullptr, T, E, k, E_loc, d, f).bytes;
}

hipError_t launch_mx_layer(const uint16_t* x, const int32_t* idx, const float* gate, int64_t T, int d,
                           int E, int k, int e_begin, int E_loc, int f, const uint8_t* const wq[3],
                           const uint8_t* const wsc[3], uint16_t* y, void* ws, hipStream_t s) {
  if (T == 0) return hipSuccess;
  const LayerWs w = carve_layer(ws, T, E, k, E_loc, d, f);
  const int64_t cap = T * std::min(k, E_loc);
  if (hipError_t e = launch_permute(x, idx, T, d, E, k, e_begin, E_loc, w.offsets, nullptr, w.row_src,
                                    w.dst, nullptr, w.perm, s);
      e != hipSuccess)
    return e;
  const FfnWs fw = carve_ffn(w.ffn, cap, E_loc, d, f, true);
  const bool small = small_tile(ceil_div(T * k * E_loc, E), E_loc, d, f);  // rows expected here
  const Scatter sc{w.dst, w.offsets, fw.tok, fw.mt, cap, k, E_loc, small ? TILE_S : TILE};
  prof_begin(K_MX_QUANT, s);
  const hipError_t e = quantize_rows(x, 1, T, d, w.xq, fw.s_perm, &sc, s);
  prof_end(K_MX_QUANT, s);
  if (e != hipSuccess) return e;
  if (hipError_t e2 = products(w.xq, T, fw.s_perm, cap, fw.tok, fw, small, w.offsets, E_loc, cap, d, f,
                               wq, wsc, w.y_perm, s);
      e2 != hipSuccess)
    return e2;
  return launch_combine(w.y_perm, w.dst, gate, T, d, k, y, s);
}

}  // namespace moe
