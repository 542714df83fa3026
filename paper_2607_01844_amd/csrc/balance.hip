// Balance loss, z-loss and per-expert counts of the router, forward and
// backward, over G groups of consecutive tokens (packed sequences; one group
// for a whole batch).  With p_t = softmax of the logits of token t, lse_t its
// log-sum-exp, n the group's valid tokens and c_e the top-k slots that chose
// expert e:
//   balance = E / (k n^2) sum_e c_e sum_t p_te,   zloss = (1 / n) sum_t lse_t^2,
//   dlogits_te = p_te (db / n (a_e - sum_e' a_e' p_te') + 2 dz / n lse_t),
//   a_e = E c_e / (k n).
// Both passes read every logit once, held in registers by a group of lanes per
// token (16 bytes a lane where rows are aligned), every load of a workgroup in
// flight at once, and are bound by that stream and its latency (few tokens: by
// the launches).  T = 65536, E = 128: 12.2 us to read the logits (33 MB), 5.5 for
// the sums over chunks, 14.6 for the gradient (67 MB); a copy of 67 MB takes 9.  Sums over tokens go through per-chunk partial
// sums in a fixed order: no floating-point atomics.
#include <algorithm>

#include "common.h"

namespace moe {
namespace {

// Over the lanes l, l ^ 1, .., of aligned groups of N lanes, in every one of them:
// within 16 lanes by lane permutations of the vector unit (mirrors serve as
// exchanges, the smaller groups being equal already), then by row and half swaps.
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
template <int N, typename F>
__device__ __forceinline__ float over_lanes(float v, F&& f) {
  if constexpr (N > 1) v = f(v, moved<0xb1>(v));    // quad_perm 1 0 3 2
  if constexpr (N > 2) v = f(v, moved<0x4e>(v));    // quad_perm 2 3 0 1
  if constexpr (N > 4) v = f(v, moved<0x141>(v));   // half a row mirrored
  if constexpr (N > 8) v = f(v, moved<0x140>(v));   // a row mirrored
  if constexpr (N > 16) {
    const auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(t[0]), __uint_as_float(t[1]));
  }
  if constexpr (N > 32) {
    const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(t[0]), __uint_as_float(t[1]));
  }
  return v;
}
struct Sum {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
// The sum over the lanes that differ in multiples of N only (the same place in
// every group of N): turns of 16 lanes, then the swaps.
template <int N, typename T>
__device__ __forceinline__ T across(T v) {
  static_assert(sizeof(T) == 4);
  auto bits = [](T a) { return __builtin_bit_cast(uint32_t, a); };
  auto val = [](uint32_t a) { return __builtin_bit_cast(T, a); };
  if constexpr (N <= 8) v += val(__builtin_amdgcn_update_dpp(0u, bits(v), 0x128, 0xf, 0xf, true));
  if constexpr (N <= 4) v += val(__builtin_amdgcn_update_dpp(0u, bits(v), 0x124, 0xf, 0xf, true));
  if constexpr (N <= 2) v += val(__builtin_amdgcn_update_dpp(0u, bits(v), 0x122, 0xf, 0xf, true));
  if constexpr (N <= 1) v += val(__builtin_amdgcn_update_dpp(0u, bits(v), 0x121, 0xf, 0xf, true));
  if constexpr (N <= 16) {
    const auto t = __builtin_amdgcn_permlane16_swap(bits(v), bits(v), false, false);
    v = val(t[0]) + val(t[1]);
  }
  if constexpr (N <= 32) {
    const auto t = __builtin_amdgcn_permlane32_swap(bits(v), bits(v), false, false);
    v = val(t[0]) + val(t[1]);
  }
  return v;
}

// A token's logits over LPR lanes: lane l holds experts 4 (l + LPR c) .. + 3,
// c < NC; experts past E read as -inf (probability 0).
template <int LPR, int NC>
struct Row {
  float v[NC][4];
  // vec: rows are 16-byte aligned (E a multiple of 4)
  __device__ __forceinline__ void load(const float* __restrict__ row, int E, int l, bool vec) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int e = 4 * (l + LPR * c);
      if (vec) {
        float4 q = make_float4(-__builtin_huge_valf(), -__builtin_huge_valf(),
                               -__builtin_huge_valf(), -__builtin_huge_valf());
        if (e < E) q = *reinterpret_cast<const float4*>(row + e);
        v[c][0] = q.x; v[c][1] = q.y; v[c][2] = q.z; v[c][3] = q.w;
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u) v[c][u] = e + u < E ? row[e + u] : -__builtin_huge_valf();
      }
    }
  }
  // v becomes exp(v - max); returns 1 / sum and the log-sum-exp.  A row of
  // -inf only (no expert left) has probabilities 0 and log-sum-exp 0.
  // The exponentials and the reciprocal are the hardware's (relative error about
  // 2^-21 for logits within 10 of the maximum, and 2^-23, beside sums in 32 bits).
  __device__ __forceinline__ void softmax(float& inv, float& lse) {
    float m = v[0][0];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int u = 0; u < 4; ++u) m = fmaxf(m, v[c][u]);
    m = over_lanes<LPR>(m, Max());
    const bool none = m == -__builtin_huge_valf();
    const float mm = none ? 0.0f : m;
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        v[c][u] = __expf(v[c][u] - mm);
        s += v[c][u];
      }
    s = over_lanes<LPR>(s, Sum());
    // a NaN row (the maximum skips NaN) keeps its NaN sum
    const bool empty = none && s == 0.0f;
    inv = empty ? 0.0f : __builtin_amdgcn_rcpf(s);
    lse = empty ? 0.0f : mm + logf(s);
  }
};

// The group that holds token t, or the next one: the first g with
// off[g + 1] > t (G: none).  A whole wave looks: 64 boundaries a step.
__device__ __forceinline__ int group_at(const int32_t* __restrict__ off, int G, int64_t t) {
  const int lane = lane_id();
  int lo = 0, n = G;
  while (n > 0) {
    const int step = (n + 63) / 64;
    const uint64_t m = __ballot(off[lo + min((lane + 1) * step, n)] > t);
    if (m == 0) return lo + n;
    const int j = static_cast<int>(__builtin_ctzll(m));
    lo += j * step;
    if (step == 1) return lo;
    n = min(step, n - j * step);
  }
  return lo;
}
// Group boundary, kept inside [0, T] (no offsets: one group of all tokens).
__device__ __forceinline__ int64_t bound(const int32_t* __restrict__ off, int g, int64_t T) {
  if (off == nullptr) return g == 0 ? 0 : T;
  const int64_t v = off[g];
  return v < 0 ? 0 : v < T ? v : T;
}

// Tokens in flight per lane of NC pieces each: eight pieces.
constexpr int in_flight(int NC) { return NC >= 8 ? 1 : 8 / NC; }

struct PartSum {
  float z;  // sum of lse^2
  int n;    // valid tokens
};

// Chunk c = tokens [c C, (c + 1) C): the part of each group g that lies in it
// goes to slot c + g (from one part to the next the chunk, the group or both
// move on, so no two parts share a slot).  Per slot: the sum of probabilities
// and the count of every expert, sum of lse^2, valid tokens.
// ONE: workgroup g takes all of group g and forms the results itself.
struct Results {
  float *balance, *zloss;
  int32_t* counts;
  float* prob_sum;
  int32_t* n_tokens;
  // the losses of group g from dot = sum_e c_e sum_t p_te
  __device__ __forceinline__ void losses(int g, int E, int k, float dot, float z, int nt) const {
    const float inv = nt > 0 ? 1.0f / static_cast<float>(nt) : 0.0f;
    balance[g] = static_cast<float>(E) / static_cast<float>(k) * (dot * inv) * inv;
    zloss[g] = z * inv;
    n_tokens[g] = nt;
  }
};
constexpr int PW = 8;  // waves
__host__ __device__ constexpr int pitch(int E) { return (E + 3) & ~3; }  // of a slot's experts
template <int LPR, int NC, bool ONE>
__global__ __launch_bounds__(64 * PW) void balance_part_kernel(
    const float* __restrict__ logits, const int32_t* __restrict__ idx,
    const int32_t* __restrict__ off, const uint8_t* __restrict__ mask, int64_t T, int E, int k,
    int G, int C, float* __restrict__ part_p, int32_t* __restrict__ part_c,
    PartSum* __restrict__ part_s, int32_t* __restrict__ ticket, Results out) {
  constexpr int R = 64 / LPR;             // tokens a wave takes at once
  constexpr int U = in_flight(NC);        // and how many times that is in flight
  constexpr int EP = 4 * LPR * NC;
  __shared__ __align__(16) float ps[PW][EP];
  __shared__ int hist[EP];
  __shared__ float zs[PW];
  __shared__ int ns[PW];
  __shared__ float ds[PW];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l = lane & (LPR - 1), r = lane / LPR;
  const bool vec = (E & 3) == 0;
  const int Ep = pitch(E);
  if constexpr (!ONE)
    for (int g = blockIdx.x * (64 * PW) + threadIdx.x; g < G; g += gridDim.x * (64 * PW)) ticket[g] = 0;
  const int64_t t0 = ONE ? 0 : static_cast<int64_t>(blockIdx.x) * C, t1 = ONE ? T : min(T, t0 + C);
  for (int g = ONE ? blockIdx.x : off == nullptr ? 0 : group_at(off, G, t0); g < G; g += ONE ? G : 1) {
    const int64_t a = max(t0, bound(off, g, T)), b = max(a, min(t1, bound(off, g + 1, T)));
    if constexpr (!ONE) {
      if (bound(off, g, T) >= t1) break;
      if (a >= b) continue;
    }
    for (int e = threadIdx.x; e < EP; e += 64 * PW) hist[e] = 0;
    // the first choices, on their way while the logits are read
    constexpr int PRE = 4;
    const int m = static_cast<int>(b - a) * k;  // at most C k
    int pre[PRE];
#pragma unroll
    for (int j = 0; j < PRE; ++j) {
      const int i = threadIdx.x + 64 * PW * j;
      const int ic = i < m ? i : m - 1;
      pre[j] = -1;
      if (ONE && m == 0) continue;
      const int e = idx[a * k + ic];
      const uint8_t there = mask == nullptr ? 1 : mask[a + ic / k];
      pre[j] = i < m && there != 0 ? e : -1;
    }
    float acc[NC][4] = {};
    float z = 0.0f, n = 0.0f;  // n: a chunk has less than 2^24 tokens
    auto take = [&](int64_t base, auto many) __attribute__((always_inline)) {
      constexpr int M = many;
      Row<LPR, NC> row[M];
      bool ok[M];
#pragma unroll
      for (int u = 0; u < M; ++u) {
        const int64_t t = base + (u * PW + w) * R + r;
        const int64_t tc = t < b ? t : b - 1;
        row[u].load(logits + tc * E, E, l, vec);
        ok[u] = t < b && (mask == nullptr || mask[tc] != 0);
      }
#pragma unroll
      for (int u = 0; u < M; ++u) {
        float inv, lse;
        row[u].softmax(inv, lse);
        if (ok[u]) {
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[c][q] = __builtin_fmaf(row[u].v[c][q], inv, acc[c][q]);
          z = __builtin_fmaf(lse, lse, z);
          n += 1.0f;
        }
      }
    };
    int64_t base = a;
    for (; base + PW * R * U <= b; base += PW * R * U) take(base, std::integral_constant<int, U>{});
    for (; base < b; base += PW * R) take(base, std::integral_constant<int, 1>{});
    // the wave's R tokens at a time, then its lanes' rows, then the waves
    if constexpr (LPR < 64) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[c][q] = across<LPR>(acc[c][q]);
      z = across<LPR>(z);
      n = across<LPR>(n);
    }
    if (lane < LPR) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
        *reinterpret_cast<float4*>(&ps[w][4 * (l + LPR * c)]) =
            make_float4(acc[c][0], acc[c][1], acc[c][2], acc[c][3]);
    }
    if (lane == 0) {
      zs[w] = z;
      ns[w] = static_cast<int>(n);
    }
    __syncthreads();  // hist is clear, the sums are there
#pragma unroll
    for (int j = 0; j < PRE; ++j)
      if (static_cast<unsigned>(pre[j]) < static_cast<unsigned>(E)) atomicAdd(&hist[pre[j]], 1);
    for (int i = threadIdx.x + 64 * PW * PRE; i < m; i += 64 * PW) {
      const int e = idx[a * k + i];
      if (static_cast<unsigned>(e) < static_cast<unsigned>(E) &&
          (mask == nullptr || mask[a + i / k] != 0))
        atomicAdd(&hist[e], 1);
    }
    __syncthreads();
    const int64_t slot = ONE ? g : static_cast<int64_t>(blockIdx.x) + g;
    float dot = 0.0f;
    for (int e = threadIdx.x; e < E; e += 64 * PW) {
      float s = ps[0][e];
#pragma unroll
      for (int q = 1; q < PW; ++q) s += ps[q][e];
      if constexpr (ONE) {
        out.prob_sum[slot * E + e] = s;
        out.counts[slot * E + e] = hist[e];
        dot = __builtin_fmaf(static_cast<float>(hist[e]), s, dot);
      } else {
        part_p[slot * Ep + e] = s;
        part_c[slot * Ep + e] = hist[e];
      }
    }
    if constexpr (ONE) {
      dot = over_lanes<64>(dot, Sum());
      if (lane == 0) ds[w] = dot;
      __syncthreads();
    }
    if (threadIdx.x == 0) {
      PartSum s{zs[0], ns[0]};
      dot = ds[0];
      for (int q = 1; q < PW; ++q) {
        s.z += zs[q];
        s.n += ns[q];
        dot += ds[q];
      }
      if constexpr (ONE) out.losses(g, E, k, dot, s.z, s.n);
      else part_s[slot] = s;
    }
    __syncthreads();
  }
}

// Group blockIdx.y, experts 32 blockIdx.x .. + 31: sums over the group's slots,
// four experts a thread and 128 slots at a time, added in an order that only
// the number of slots decides.  The last workgroup of a group to finish (by a
// ticket) adds the groups of 32 experts and forms the losses.
constexpr int RE = 32, RW = 16;  // experts, waves
// Writes v where every workgroup sees it before any later access of this lane:
// the exchange has returned.  (A fence would write whole caches back.)
__device__ __forceinline__ void put_first(float* at, float v) {
  const float old = __hip_atomic_exchange(at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  asm volatile("" ::"v"(old) : "memory");
}
__global__ __launch_bounds__(64 * RW) void balance_reduce_kernel(
    const float* __restrict__ part_p, const int32_t* __restrict__ part_c,
    const PartSum* __restrict__ part_s, const int32_t* __restrict__ off, int64_t T, int E, int k,
    int C, float* __restrict__ dots, int32_t* __restrict__ ticket, Results out) {
  __shared__ __align__(16) float fs[RW][RE];
  __shared__ __align__(16) int is[RW][RE];
  __shared__ float zs[RW];
  __shared__ int ns[RW];
  const int g = blockIdx.y, EB = gridDim.x, Ep = pitch(E);  // EB at most 32: E at most 1024
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int e4 = blockIdx.x * RE + 4 * (lane & 7);
  const int64_t a = bound(off, g, T), b = bound(off, g + 1, T);
  const int64_t s0 = a / C + g, s1 = a < b ? (b - 1) / C + g + 1 : s0;
  float p[4] = {};
  int n[4] = {};
  if (e4 < Ep) {
#pragma unroll 4
    for (int64_t s = s0 + (threadIdx.x >> 3); s < s1; s += 8 * RW) {
      const float4 v = *reinterpret_cast<const float4*>(part_p + s * Ep + e4);
      const int4 c = *reinterpret_cast<const int4*>(part_c + s * Ep + e4);
      p[0] += v.x; p[1] += v.y; p[2] += v.z; p[3] += v.w;
      n[0] += c.x; n[1] += c.y; n[2] += c.z; n[3] += c.w;
    }
  }
  float z = 0.0f;  // sum of lse^2 and the valid tokens
  int nt = 0;
  for (int64_t s = s0 + threadIdx.x; s < s1; s += 64 * RW) {
    z += part_s[s].z;
    nt += part_s[s].n;
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    p[u] = across<8>(p[u]);
    n[u] = across<8>(n[u]);
  }
  z = across<1>(z);
  nt = across<1>(nt);
  if (lane < 8) {
    *reinterpret_cast<float4*>(&fs[w][4 * lane]) = make_float4(p[0], p[1], p[2], p[3]);
    *reinterpret_cast<int4*>(&is[w][4 * lane]) = make_int4(n[0], n[1], n[2], n[3]);
  }
  if (lane == 0) {
    zs[w] = z;
    ns[w] = nt;
  }
  __syncthreads();
  if (w != 0) return;
  const int q = lane & (RE - 1), e = blockIdx.x * RE + q;
  float ps = fs[0][q];
  int cs = is[0][q];
  z = zs[0];
  nt = ns[0];
#pragma unroll
  for (int i = 1; i < RW; ++i) {
    ps += fs[i][q];
    cs += is[i][q];
    z += zs[i];
    nt += ns[i];
  }
  if (e < E && lane < RE) {
    out.counts[static_cast<int64_t>(g) * E + e] = cs;
    out.prob_sum[static_cast<int64_t>(g) * E + e] = ps;
  }
  float dot = over_lanes<RE>(e < E ? static_cast<float>(cs) * ps : 0.0f, Sum());
  if (EB > 1) {
    float* const dg = dots + static_cast<int64_t>(g) * EB;
    int at = 0;
    if (lane == 0) {
      put_first(dg + blockIdx.x, dot);
      at = __hip_atomic_fetch_add(&ticket[g], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (__builtin_amdgcn_readfirstlane(at) != EB - 1) return;
    dot = lane < EB ? __hip_atomic_load(dg + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0f;
    dot = over_lanes<RE>(dot, Sum());
  }
  if (lane == 0) out.losses(g, E, k, dot, z, nt);
}

// Logit gradients of BC tokens a workgroup of BW waves.  Tokens outside every group, masked
// ones and those of a group of no valid tokens get 0 (accumulate: are left).
constexpr int BW = 4;
template <int LPR, int NC>
__global__ __launch_bounds__(64 * BW) void balance_bwd_kernel(
    const float* __restrict__ logits, const int32_t* __restrict__ off,
    const uint8_t* __restrict__ mask, const int32_t* __restrict__ counts,
    const int32_t* __restrict__ n_tokens, const float* __restrict__ dbalance,
    const float* __restrict__ dzloss, int64_t T, int E, int k, int G, int BC,
    int accumulate, float* __restrict__ dlogits) {
  constexpr int R = 64 / LPR;
  constexpr int U = in_flight(NC);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l = lane & (LPR - 1), r = lane / LPR;
  const bool vec = (E & 3) == 0;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * BC, t1 = min(T, t0 + BC);
  int64_t at = t0;  // tokens before it are done
  int g = off == nullptr ? 0 : group_at(off, G, t0);
  while (at < t1) {
    // the next part: of group g, or (outside) up to the next group's start
    int64_t b = t1;
    bool inside = false;
    if (g < G) {
      const int64_t a = bound(off, g, T);
      if (a > at) {
        b = min(t1, a);
      } else {
        b = min(t1, bound(off, g + 1, T));
        inside = true;
        if (b <= at) {
          ++g;
          continue;
        }
      }
    }
    float fb = 0.0f, fz = 0.0f;
    if (inside) {
      const int n = n_tokens[g];
      const float inv = n > 0 ? 1.0f / static_cast<float>(n) : 0.0f;
      fb = dbalance[g] * inv * (static_cast<float>(E) / static_cast<float>(k) * inv);
      fz = 2.0f * dzloss[g] * inv;
    }
    const int32_t* const cg = counts + static_cast<int64_t>(inside ? g : 0) * E;
    auto take = [&](int64_t base, auto many) __attribute__((always_inline)) {
      constexpr int M = many;
      Row<LPR, NC> row[M];
      bool ok[M];
#pragma unroll
      for (int u = 0; u < M; ++u) {
        const int64_t t = base + (u * BW + w) * R + r;
        const int64_t tc = t < b ? t : b - 1;
        row[u].load(logits + tc * E, E, l, vec);
        ok[u] = t < b && inside && (mask == nullptr || mask[tc] != 0);
      }
      // a part is seldom more than one step: its counts come with the logits
      float ae[NC][4];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int e = 4 * (l + LPR * c);
        if (vec) {
          int4 q = make_int4(0, 0, 0, 0);
          if (e < E) q = *reinterpret_cast<const int4*>(cg + e);
          ae[c][0] = fb * static_cast<float>(q.x);
          ae[c][1] = fb * static_cast<float>(q.y);
          ae[c][2] = fb * static_cast<float>(q.z);
          ae[c][3] = fb * static_cast<float>(q.w);
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) ae[c][q] = e + q < E ? fb * static_cast<float>(cg[e + q]) : 0.0f;
        }
      }
#pragma unroll
      for (int u = 0; u < M; ++u) {
        const int64_t t = base + (u * BW + w) * R + r;
        float inv, lse;
        row[u].softmax(inv, lse);
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            row[u].v[c][q] *= inv;
            s = __builtin_fmaf(ae[c][q], row[u].v[c][q], s);
          }
        s = over_lanes<LPR>(s, Sum());
        const float add = __builtin_fmaf(fz, lse, -s);
        if (t >= b || (accumulate && !ok[u])) continue;
        float* out = dlogits + t * E;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const int e = 4 * (l + LPR * c);
          float d[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) d[q] = ok[u] ? row[u].v[c][q] * (ae[c][q] + add) : 0.0f;
          if (vec) {
            if (e >= E) continue;
            float4* o = reinterpret_cast<float4*>(out + e);
            if (accumulate) {
              const float4 h = *o;
              d[0] += h.x; d[1] += h.y; d[2] += h.z; d[3] += h.w;
            }
            *o = make_float4(d[0], d[1], d[2], d[3]);
          } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
              if (e + q < E) out[e + q] = accumulate ? out[e + q] + d[q] : d[q];
          }
        }
      }
    };
    int64_t base = at;
    for (; base + BW * R * U <= b; base += BW * R * U) take(base, std::integral_constant<int, U>{});
    for (; base < b; base += BW * R) take(base, std::integral_constant<int, 1>{});
    at = b;
  }
}

// Calls f with the lanes per row and 16-byte pieces per lane that hold E
// experts: eight lanes where they do with four pieces (lines of 128 bytes, and
// few steps between lanes), more from there on.
template <typename F>
hipError_t with_shape(int E, F&& f) {
  auto go = [&](auto L, auto N) { return f(L, N); };
#define MOE_SHAPE(L, N) return go(std::integral_constant<int, L>{}, std::integral_constant<int, N>{})
  const int need = (E + 3) / 4;
  if (need <= 1) MOE_SHAPE(1, 1);
  if (need <= 2) MOE_SHAPE(2, 1);
  if (need <= 4) MOE_SHAPE(4, 1);
  if (need <= 8) MOE_SHAPE(8, 1);
  if (need <= 16) MOE_SHAPE(8, 2);
  if (need <= 24) MOE_SHAPE(8, 3);
  if (need <= 32) MOE_SHAPE(8, 4);
  if (need <= 48) MOE_SHAPE(16, 3);
  if (need <= 64) MOE_SHAPE(16, 4);
  if (need <= 96) MOE_SHAPE(32, 3);
  if (need <= 128) MOE_SHAPE(32, 4);
  if (need <= 192) MOE_SHAPE(64, 3);
  MOE_SHAPE(64, 4);
#undef MOE_SHAPE
}

// Tokens of a chunk: two workgroups per compute unit and at least 32 tokens.
// T = 16384, E = 384, 13 sequences: the pass over the logits takes 13.9 us, with
// 256 chunks 17.6; twice the chunks cost the sums over them 1.5 us and gain none.
int part_chunk(int64_t T) {
  return static_cast<int>(align_up(static_cast<size_t>(std::max<int64_t>(32, ceil_div(T, 512))), 32));
}
// Few logits (64 KiB, what a workgroup reads in about a microsecond): a workgroup
// per group and one launch instead of two, each 4 us of a small call.
bool few(int64_t T, int E) { return T * E <= 16384; }

}  // namespace

size_t balance_ws_bytes(int64_t T, int E, int G) {
  const size_t slots = static_cast<size_t>(ceil_div(T, part_chunk(T))) + G;
  return 2 * align_up(sizeof(float) * slots * pitch(E), 256) + align_up(sizeof(PartSum) * slots, 256) +
         align_up(sizeof(float) * static_cast<size_t>(G) * ceil_div(E, RE), 256) +
         align_up(sizeof(int32_t) * static_cast<size_t>(G), 256);
}

hipError_t launch_balance_fwd(const float* logits, const int32_t* idx, const int32_t* off,
                              const uint8_t* mask, int64_t T, int E, int k, int G, float* balance,
                              float* zloss, int32_t* counts, float* prob_sum, int32_t* n_tokens,
                              void* ws, hipStream_t s) {
  const Results out{balance, zloss, counts, prob_sum, n_tokens};
  if (few(T, E)) {
    prof_begin(K_BALANCE_PART, s);
    const hipError_t e = with_shape(E, [&](auto L, auto N) {
      balance_part_kernel<L, N, true><<<static_cast<unsigned>(G), 64 * PW, 0, s>>>(
          logits, idx, off, mask, T, E, k, G, 0, nullptr, nullptr, nullptr, nullptr, out);
      return hipGetLastError();
    });
    prof_end(K_BALANCE_PART, s);
    return e;
  }
  const int C = part_chunk(T);
  const int64_t chunks = ceil_div(T, C);
  const size_t slots = static_cast<size_t>(chunks) + G;
  char* p = static_cast<char*>(ws);
  float* part_p = reinterpret_cast<float*>(p);
  p += align_up(sizeof(float) * slots * pitch(E), 256);
  int32_t* part_c = reinterpret_cast<int32_t*>(p);
  p += align_up(sizeof(int32_t) * slots * pitch(E), 256);
  PartSum* part_s = reinterpret_cast<PartSum*>(p);
  p += align_up(sizeof(PartSum) * slots, 256);
  float* dots = reinterpret_cast<float*>(p);
  p += align_up(sizeof(float) * static_cast<size_t>(G) * ceil_div(E, RE), 256);
  int32_t* ticket = reinterpret_cast<int32_t*>(p);
  prof_begin(K_BALANCE_PART, s);
  const hipError_t e = with_shape(E, [&](auto L, auto N) {
    balance_part_kernel<L, N, false><<<static_cast<unsigned>(chunks), 64 * PW, 0, s>>>(
        logits, idx, off, mask, T, E, k, G, C, part_p, part_c, part_s, ticket, out);
    return hipGetLastError();
  });
  prof_end(K_BALANCE_PART, s);
  if (e != hipSuccess) return e;
  prof_begin(K_BALANCE_SUM, s);
  balance_reduce_kernel<<<dim3(static_cast<unsigned>(ceil_div(E, RE)), static_cast<unsigned>(G)),
                          64 * RW, 0, s>>>(part_p, part_c, part_s, off, T, E, k, C, dots, ticket, out);
  prof_end(K_BALANCE_SUM, s);
  return hipGetLastError();
}

hipError_t launch_balance_bwd(const float* logits, const int32_t* off, const uint8_t* mask,
                              const int32_t* counts, const int32_t* n_tokens,
                              const float* dbalance, const float* dzloss, int64_t T, int E, int k,
                              int G, int accumulate, float* dlogits, hipStream_t s) {
  if (T == 0) return hipSuccess;
  prof_begin(K_BALANCE_BWD, s);
  const hipError_t e = with_shape(E, [&](auto L, auto N) {
    // every load of a workgroup in flight at once; fewer a workgroup where that
    // would leave compute units without one
    constexpr int one = BW * (64 / decltype(L)::value), all = one * in_flight(decltype(N)::value);
    const int BC = T >= 256 * all ? all : one;
    balance_bwd_kernel<L, N><<<static_cast<unsigned>(ceil_div(T, BC)), 64 * BW, 0, s>>>(
        logits, off, mask, counts, n_tokens, dbalance, dzloss, T, E, k, G, BC, accumulate, dlogits);
    return hipGetLastError();
  });
  prof_end(K_BALANCE_BWD, s);
  return e;
}

}  // namespace moe
