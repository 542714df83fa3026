// Layer norm of rows of bf16, forward (with the residual sum) and backward (gfx950).
//   h = bf16(x + residual), mu = mean h, r = 1 / sqrt(mean (h - mu)^2 + eps),
//   y = (h - mu) r gamma + beta;
//   with xh = (h - mu) r and g = dy gamma:
//   dx = dh + r (g - mean g - xh mean(g xh)), dgamma = sum_t dy xh, dbeta = sum_t dy.
// A row is held in registers by W waves, so each operand crosses HBM once; the
// mean is subtracted before the squares are summed (a row far from zero keeps its
// variance).  Sums, statistics and the weights' gradients are fp32; every
// bf16 result is rounded once.  Bound by the HBM stream: T = 65536, d = 4096 with the
// residual, 2.15 GB each way, forward 380 us, 5.6 TB/s, backward 373, 5.75; few rows by
// latency (16 of them: 3.4 us).
#include <algorithm>

#include "common.h"

namespace moe {
namespace {

__device__ __forceinline__ uint4 add8(const uint4& a, const uint4& b) {
  float f[8], g[8];
  unpack8(a, f);
  unpack8(b, g);
#pragma unroll
  for (int q = 0; q < 8; ++q) f[q] += g[q];
  return pack8(f);
}
__device__ __forceinline__ void load8f(const float* __restrict__ p, float* f) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}

template <bool STREAM>
__device__ __forceinline__ uint4 load_row(const uint4* p) {
  if constexpr (STREAM) return load_stream(p);
  else return *p;
}

// Over the W waves of a row: the sums of n values, in every lane.  `red` is this
// exchange's own place; with two exchanges a round, one barrier each is enough.
template <int W, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* red, int w, int lane) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = over_lanes<64>(v[i], Sum());
  if constexpr (W > 1) {
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) red[i * W + w] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = red[i * W];
#pragma unroll
      for (int u = 1; u < W; ++u) v[i] += red[i * W + u];
    }
  }
}

// Waves of a row W, chunks of 8 columns a lane C; chunk c of lane l of wave w is
// (c W + w) 64 + l.  STREAM: loads that no cache keeps.
template <int W, int C, bool RES, bool STREAM>
__global__ __launch_bounds__(W < 4 ? 256 : 64 * W) void norm_fwd_kernel(
    const uint16_t* __restrict__ x, const uint16_t* __restrict__ res,
    const float* __restrict__ gamma, const float* __restrict__ beta, int64_t T, int d, float eps,
    uint16_t* __restrict__ h, uint16_t* __restrict__ y, float* __restrict__ mean,
    float* __restrict__ rstd) {
  constexpr int G = W < 4 ? 4 / W : 1;  // rows' teams of a workgroup
  __shared__ float red[2][W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int w = wave % W, team = wave / W;
  const int nch = d >> 3;
  const float fd = static_cast<float>(d);
  float ga[C][8], be[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (c * W + w) * 64 + lane;
#pragma unroll
    for (int q = 0; q < 8; ++q) be[c][q] = 0.0f;
    if (at < nch) {
      load8f(gamma + 8 * at, ga[c]);
      if (beta) load8f(beta + 8 * at, be[c]);
    }
  }
  const int64_t step = static_cast<int64_t>(gridDim.x) * G;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * G + team; t < T; t += step) {
    uint4 v[C], e[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (c * W + w) * 64 + lane;
      v[c] = make_uint4(0, 0, 0, 0);
      if (at < nch) {
        v[c] = load_row<STREAM>(reinterpret_cast<const uint4*>(x + t * d) + at);
        if constexpr (RES) e[c] = load_row<STREAM>(reinterpret_cast<const uint4*>(res + t * d) + at);
      }
    }
    if constexpr (RES) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int at = (c * W + w) * 64 + lane;
        if (at < nch) {
          v[c] = add8(v[c], e[c]);
          store_stream(reinterpret_cast<uint4*>(h + t * d) + at, v[c]);
        }
      }
    }
    float mu[1] = {0.0f}, sq[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float f[8];
      unpack8(v[c], f);
#pragma unroll
      for (int q = 0; q < 8; ++q) mu[0] += f[q];
    }
    row_sums<W>(mu, red[0], w, lane);
    mu[0] /= fd;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float f[8];
      unpack8(v[c], f);
      if ((c * W + w) * 64 + lane < nch)
#pragma unroll
        for (int q = 0; q < 8; ++q) sq[0] += (f[q] - mu[0]) * (f[q] - mu[0]);
    }
    row_sums<W>(sq, red[1], w, lane);
    const float rs = 1.0f / sqrtf(sq[0] / fd + eps);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (c * W + w) * 64 + lane;
      float f[8];
      unpack8(v[c], f);
#pragma unroll
      for (int q = 0; q < 8; ++q) f[q] = (f[q] - mu[0]) * rs * ga[c][q] + be[c][q];
      if (at < nch) store_stream(reinterpret_cast<uint4*>(y + t * d) + at, pack8(f));
    }
    if (w == 0 && lane == 0) {
      if (mean) mean[t] = mu[0];
      if (rstd) rstd[t] = rs;
    }
  }
}

// part [workgroups][2][d]: the workgroup's sums of dy xh and of dy.  dx may lie in the
// memory of dy, h or dh (so these promise nothing of each other): every thread reads
// what it overwrites before, and nothing else is read there.
template <int W, int C, bool DH, bool STREAM>
__global__ __launch_bounds__(W < 4 ? 256 : 64 * W) void norm_bwd_kernel(
    const uint16_t* dy, const uint16_t* h, const float* __restrict__ gamma,
    const float* __restrict__ mean, const float* __restrict__ rstd, const uint16_t* dh, int64_t T,
    int d, uint16_t* dx, float* __restrict__ part) {
  constexpr int G = W < 4 ? 4 / W : 1;
  __shared__ float red[2][2 * W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int w = wave % W, team = wave / W;
  const int nch = d >> 3;
  const float fd = static_cast<float>(d);
  float ga[C][8], dg[C][8], db[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (c * W + w) * 64 + lane;
#pragma unroll
    for (int q = 0; q < 8; ++q) ga[c][q] = dg[c][q] = db[c][q] = 0.0f;
    if (at < nch) load8f(gamma + 8 * at, ga[c]);
  }
  const int64_t step = static_cast<int64_t>(gridDim.x) * G;
  int turn = 0;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * G + team; t < T; t += step) {
    uint4 a[C], b[C], e[C];
    const float mu = mean[t], rs = rstd[t];
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (c * W + w) * 64 + lane;
      a[c] = b[c] = make_uint4(0, 0, 0, 0);
      if (at < nch) {
        a[c] = load_row<STREAM>(reinterpret_cast<const uint4*>(dy + t * d) + at);
        b[c] = load_row<STREAM>(reinterpret_cast<const uint4*>(h + t * d) + at);
        if constexpr (DH) e[c] = load_row<STREAM>(reinterpret_cast<const uint4*>(dh + t * d) + at);
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if ((c * W + w) * 64 + lane < nch) {
        float f[8], g[8];
        unpack8(a[c], g);
        unpack8(b[c], f);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const float xh = (f[q] - mu) * rs;
          dg[c][q] += g[q] * xh;
          db[c][q] += g[q];
          s[0] += g[q] * ga[c][q];
          s[1] += g[q] * ga[c][q] * xh;
        }
      }
    }
    // two places by turns: a wave may be a round ahead of another's reads
    row_sums<W>(s, red[turn], w, lane);
    turn ^= 1;
    const float m1 = s[0] / fd, m2 = s[1] / fd;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (c * W + w) * 64 + lane;
      float f[8], g[8];
      unpack8(a[c], g);
      unpack8(b[c], f);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float xh = (f[q] - mu) * rs;
        f[q] = (g[q] * ga[c][q] - m1 - xh * m2) * rs;
      }
      if constexpr (DH) {
        unpack8(e[c], g);
#pragma unroll
        for (int q = 0; q < 8; ++q) f[q] += g[q];
      }
      if (at < nch) {
        uint4* o = reinterpret_cast<uint4*>(dx + t * d) + at;
        if constexpr (STREAM) store_stream(o, pack8(f));
        else *o = pack8(f);
      }
    }
  }
  float* p = part + static_cast<int64_t>(blockIdx.x) * 2 * d;
  if constexpr (G == 1) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (c * W + w) * 64 + lane;
      if (at < nch)
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          p[8 * at + q] = dg[c][q];
          p[d + 8 * at + q] = db[c][q];
        }
    }
  } else {
    // the teams' sums, in their order
    static_assert(W == 1, "a team's columns are those of one wave");
    __shared__ float sums[G][C * 64 * 8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (k) __syncthreads();
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int q = 0; q < 8; ++q)
          sums[team][(c * 64 + lane) * 8 + q] = k ? db[c][q] : dg[c][q];
      __syncthreads();
      for (int i = threadIdx.x; i < d; i += 256) {
        float v = sums[0][i];
#pragma unroll
        for (int g = 1; g < G; ++g) v += sums[g][i];
        p[k * d + i] = v;
      }
    }
  }
}

// Rows beyond the registers' reach (d > NORM_HELD): a workgroup of 16 waves walks
// its row again for each sum (its second and third passes come from the caches).
template <bool RES>
__global__ __launch_bounds__(1024) void norm_fwd_long_kernel(
    const uint16_t* __restrict__ x, const uint16_t* __restrict__ res,
    const float* __restrict__ gamma, const float* __restrict__ beta, int64_t T, int d, float eps,
    uint16_t* __restrict__ h, uint16_t* __restrict__ y, float* __restrict__ mean,
    float* __restrict__ rstd) {
  __shared__ float red[2][16];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nch = d >> 3;
  const float fd = static_cast<float>(d);
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
    const uint4* row = reinterpret_cast<const uint4*>(x + t * d);
    float s[1] = {0.0f}, sq[1] = {0.0f}, f[8];
    for (int c = threadIdx.x; c < nch; c += 1024) {
      uint4 v = row[c];
      if constexpr (RES) {
        v = add8(v, reinterpret_cast<const uint4*>(res + t * d)[c]);
        reinterpret_cast<uint4*>(h + t * d)[c] = v;
      }
      unpack8(v, f);
#pragma unroll
      for (int q = 0; q < 8; ++q) s[0] += f[q];
    }
    // each thread reads again what it wrote itself
    if constexpr (RES) row = reinterpret_cast<const uint4*>(h + t * d);
    row_sums<16>(s, red[0], w, lane);
    const float mu = s[0] / fd;
    for (int c = threadIdx.x; c < nch; c += 1024) {
      unpack8(row[c], f);
#pragma unroll
      for (int q = 0; q < 8; ++q) sq[0] += (f[q] - mu) * (f[q] - mu);
    }
    row_sums<16>(sq, red[1], w, lane);
    const float rs = 1.0f / sqrtf(sq[0] / fd + eps);
    for (int c = threadIdx.x; c < nch; c += 1024) {
      float ga[8], be[8];
      unpack8(row[c], f);
      load8f(gamma + 8 * c, ga);
#pragma unroll
      for (int q = 0; q < 8; ++q) be[q] = 0.0f;
      if (beta) load8f(beta + 8 * c, be);
#pragma unroll
      for (int q = 0; q < 8; ++q) f[q] = (f[q] - mu) * rs * ga[q] + be[q];
      reinterpret_cast<uint4*>(y + t * d)[c] = pack8(f);
    }
    if (threadIdx.x == 0) {
      if (mean) mean[t] = mu;
      if (rstd) rstd[t] = rs;
    }
  }
}

template <bool DH>
__global__ __launch_bounds__(1024) void norm_bwd_long_kernel(
    const uint16_t* dy, const uint16_t* h, const float* __restrict__ gamma,
    const float* __restrict__ mean, const float* __restrict__ rstd, const uint16_t* dh, int64_t T,
    int d, uint16_t* dx) {
  __shared__ float red[2][32];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nch = d >> 3;
  const float fd = static_cast<float>(d);
  int turn = 0;
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
    const uint4* row = reinterpret_cast<const uint4*>(h + t * d);
    const uint4* up = reinterpret_cast<const uint4*>(dy + t * d);
    const float mu = mean[t], rs = rstd[t];
    float s[2] = {0.0f, 0.0f}, f[8], g[8], ga[8];
    for (int c = threadIdx.x; c < nch; c += 1024) {
      unpack8(row[c], f);
      unpack8(up[c], g);
      load8f(gamma + 8 * c, ga);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        s[0] += g[q] * ga[q];
        s[1] += g[q] * ga[q] * ((f[q] - mu) * rs);
      }
    }
    row_sums<16>(s, red[turn], w, lane);
    turn ^= 1;
    const float m1 = s[0] / fd, m2 = s[1] / fd;
    for (int c = threadIdx.x; c < nch; c += 1024) {
      unpack8(row[c], f);
      unpack8(up[c], g);
      load8f(gamma + 8 * c, ga);
#pragma unroll
      for (int q = 0; q < 8; ++q) f[q] = (g[q] * ga[q] - m1 - (f[q] - mu) * rs * m2) * rs;
      if constexpr (DH) {
        unpack8(reinterpret_cast<const uint4*>(dh + t * d)[c], g);
#pragma unroll
        for (int q = 0; q < 8; ++q) f[q] += g[q];
      }
      reinterpret_cast<uint4*>(dx + t * d)[c] = pack8(f);
    }
  }
}
// Its weights' gradients: a wave sums 512 columns over a part of the rows.
__global__ __launch_bounds__(256) void norm_cols_kernel(
    const uint16_t* __restrict__ dy, const uint16_t* __restrict__ h,
    const float* __restrict__ mean, const float* __restrict__ rstd, int64_t T, int d, int64_t rows,
    float* __restrict__ part) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = (blockIdx.x * 4 + w) * 64 + lane;
  if (c >= d >> 3) return;
  float dg[8] = {}, db[8] = {}, f[8], g[8];
  const int64_t t1 = min(T, (blockIdx.y + 1) * rows);
  for (int64_t t = blockIdx.y * rows; t < t1; ++t) {
    unpack8(reinterpret_cast<const uint4*>(h + t * d)[c], f);
    unpack8(reinterpret_cast<const uint4*>(dy + t * d)[c], g);
    const float mu = mean[t], rs = rstd[t];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      dg[q] += g[q] * ((f[q] - mu) * rs);
      db[q] += g[q];
    }
  }
  float* p = part + static_cast<int64_t>(blockIdx.y) * 2 * d + 8 * c;
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    p[q] = dg[q];
    p[d + q] = db[q];
  }
}

// out[i] = sum over parts of part[p][i]: 64 columns a workgroup, its 16 waves take
// every 16th part (joined in order), dgamma then dbeta (null: not wanted).
constexpr int SUM_W = 16;
__global__ __launch_bounds__(64 * SUM_W) void norm_sum_kernel(const float* __restrict__ part,
                                                              int parts, int d,
                                                              float* __restrict__ dgamma,
                                                              float* __restrict__ dbeta) {
  __shared__ float sums[SUM_W][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 64 + lane, pitch = 2 * static_cast<int64_t>(d);
  constexpr int B = 8;
  float s = 0.0f;
  if (i < pitch) {
    int p = w;
    for (; p + (B - 1) * SUM_W < parts; p += B * SUM_W) {
      float v[B];
#pragma unroll
      for (int u = 0; u < B; ++u) v[u] = part[(p + u * SUM_W) * pitch + i];
#pragma unroll
      for (int u = 0; u < B; ++u) s += v[u];
    }
    for (; p < parts; p += SUM_W) s += part[p * pitch + i];
  }
  sums[w][lane] = s;
  __syncthreads();
  if (w == 0 && i < pitch) {
    for (int u = 1; u < SUM_W; ++u) s += sums[u][lane];
    if (i < d)
      dgamma[i] = s;
    else if (dbeta)
      dbeta[i - d] = s;
  }
}

constexpr int NORM_HELD = 16384;  // widest row held in registers

// Two workgroups a compute unit walk the rows (three of narrow rows, one of 16 waves in
// the backward pass): few rows in flight, far apart, suit HBM best (T = 65536, d = 4096,
// 2.15 GB each way: forward 424 us on 256 workgroups, 381 on 512, 388 on 768, 398 on
// 2048; backward 431, 376, 438, 444; d = 512: 43 on 512, 42 on 768, and 46, 45).
// A backward pass has fewer where a team would get under 16 rows: its partial sums,
// 8 bytes a column, weigh against 6 or 8 a row's (T = 4096, d = 8192: 63 us on 256
// workgroups, 72 on 512, 91 on 1024).
int64_t groups_a_cu(int d) { return d <= 1024 ? 3 : 2; }
int64_t bwd_groups(int64_t T, int d) {
  if (T == 0) return 1;
  if (d > NORM_HELD) return std::clamp<int64_t>(T / 64, 1, 64);
  const int64_t teams = d <= 2048 ? 4 : 1, most = d <= 8192 ? 256 * groups_a_cu(d) : 256;
  const int64_t rows = std::max(ceil_div(T, teams * most),
                                std::min<int64_t>(16, ceil_div(T, teams * 256)));  // of a team
  return std::max<int64_t>(1, ceil_div(T, teams * rows));
}

// Calls that move this much gain from keeping their reads out of the caches (and the
// backward's dx): forward of 2.15 GB 401 -> 381 us, backward 401 -> 376, of 470 MB
// 94 -> 89; less may find its inputs there (forward of 470 MB 70 us, with streamed loads
// 81, of 268 MB 42 and 48; backward of 268 MB 51 and 58).  y and h are streamed always
// (2.15 GB: 397 -> 381 us, 268 MB: 43 to 45 -> 42).
constexpr int64_t STREAM_FWD = int64_t{768} << 20, STREAM_BWD = int64_t{384} << 20;

// A wave a row up to 2048 columns (32 registers of it a lane), then eight and sixteen.
template <typename F>
void by_width(int d, F&& f) {
  using std::integral_constant;
  if (d <= 512) f(integral_constant<int, 1>{}, integral_constant<int, 1>{});
  else if (d <= 1024) f(integral_constant<int, 1>{}, integral_constant<int, 2>{});
  else if (d <= 2048) f(integral_constant<int, 1>{}, integral_constant<int, 4>{});
  else if (d <= 4096) f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
  else if (d <= 8192) f(integral_constant<int, 8>{}, integral_constant<int, 2>{});
  else f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
}
// f(true_type) or f(false_type)
template <typename F>
void either(bool v, F&& f) {
  if (v) f(std::true_type{});
  else f(std::false_type{});
}

}  // namespace

hipError_t launch_norm_fwd(const uint16_t* x, const uint16_t* res, const float* gamma,
                           const float* beta, int64_t T, int d, float eps, uint16_t* h,
                           uint16_t* y, float* mean, float* rstd, hipStream_t s) {
  if (T == 0) return hipSuccess;
  prof_begin(K_NORM_FWD, s);
  if (d > NORM_HELD) {
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(T, 2 * device_cus()));
    if (res)
      norm_fwd_long_kernel<true><<<grid, 1024, 0, s>>>(x, res, gamma, beta, T, d, eps, h, y, mean, rstd);
    else
      norm_fwd_long_kernel<false><<<grid, 1024, 0, s>>>(x, res, gamma, beta, T, d, eps, h, y, mean, rstd);
  } else {
    const bool stream = T * d * (res ? 8 : 4) >= STREAM_FWD;
    by_width(d, [&](auto w, auto c) {
      constexpr int W = w, C = c, G = W < 4 ? 4 / W : 1, threads = W < 4 ? 256 : 64 * W;
      // one load of 16 bytes a lane and row is too little in flight (T = 65536, d = 4096
      // without the residual: 217 us, with twice the workgroups 191)
      const int more = !res && W > 1 && C == 1 ? 2 : 1;
      const unsigned grid = static_cast<unsigned>(
          std::min<int64_t>(ceil_div(T, G), more * groups_a_cu(d) * device_cus()));
      either(res != nullptr, [&](auto r) {
        either(stream, [&](auto st) {
          norm_fwd_kernel<W, C, r, st><<<grid, threads, 0, s>>>(x, res, gamma, beta, T, d, eps, h,
                                                                y, mean, rstd);
        });
      });
    });
  }
  prof_end(K_NORM_FWD, s);
  return hipGetLastError();
}

size_t norm_bwd_ws_bytes(int64_t T, int d) {
  return align_up(sizeof(float) * 2 * static_cast<size_t>(bwd_groups(T, d)) * d, 256);
}

hipError_t launch_norm_bwd(const uint16_t* dy, const uint16_t* h, const float* gamma,
                           const float* mean, const float* rstd, const uint16_t* dh, int64_t T,
                           int d, uint16_t* dx, float* dgamma, float* dbeta, void* ws,
                           hipStream_t s) {
  float* part = static_cast<float*>(ws);
  const int64_t groups = T == 0 ? 0 : bwd_groups(T, d);
  if (T > 0) {
    prof_begin(K_NORM_BWD, s);
    if (d > NORM_HELD) {
      // the columns' sums first: dx may lie in the memory of dy or h
      const dim3 cols(static_cast<unsigned>(ceil_div(d, 2048)), static_cast<unsigned>(groups));
      norm_cols_kernel<<<cols, 256, 0, s>>>(dy, h, mean, rstd, T, d, ceil_div(T, groups), part);
      const unsigned grid = static_cast<unsigned>(std::min<int64_t>(T, 2 * device_cus()));
      if (dh)
        norm_bwd_long_kernel<true><<<grid, 1024, 0, s>>>(dy, h, gamma, mean, rstd, dh, T, d, dx);
      else
        norm_bwd_long_kernel<false><<<grid, 1024, 0, s>>>(dy, h, gamma, mean, rstd, dh, T, d, dx);
    } else {
      const bool stream = T * d * (dh ? 8 : 6) >= STREAM_BWD;
      by_width(d, [&](auto w, auto c) {
        constexpr int W = w, C = c, threads = W < 4 ? 256 : 64 * W;
        either(dh != nullptr, [&](auto r) {
          either(stream, [&](auto st) {
            norm_bwd_kernel<W, C, r, st><<<static_cast<unsigned>(groups), threads, 0, s>>>(
                dy, h, gamma, mean, rstd, dh, T, d, dx, part);
          });
        });
      });
    }
    prof_end(K_NORM_BWD, s);
  }
  prof_begin(K_NORM_SUM, s);
  norm_sum_kernel<<<static_cast<unsigned>(ceil_div(2 * static_cast<int64_t>(d), 64)), 64 * SUM_W, 0, s>>>(
      part, static_cast<int>(groups), d, dgamma, dbeta);
  prof_end(K_NORM_SUM, s);
  return hipGetLastError();
}

}  // namespace moe
