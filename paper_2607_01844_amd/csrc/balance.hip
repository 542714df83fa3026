// Balance loss, z-loss and per-expert counts of the router, forward and
// backward, over G groups of consecutive tokens (packed sequences; one group
// for a whole batch).  With p_t = softmax of the logits of token t, lse_t its
// log-sum-exp, n the group's valid tokens and c_e the top-k slots that chose
// expert e:
//   balance = E / (k n^2) sum_e c_e sum_t p_te,   zloss = (1 / n) sum_t lse_t^2,
//   dlogits_te = p_te (db / n (a_e - sum_e' a_e' p_te') + 2 dz / n lse_t),
//   a_e = E c_e / (k n).
// Both passes read every logit once, held in registers by a group of lanes per
// token (16 bytes a lane where rows are aligned), and are bound by that stream
// (few tokens: by the launches).  Sums over tokens go through per-chunk partial
// sums in a fixed order: no floating-point atomics.
#include <algorithm>

#include "common.h"

namespace moe {
namespace {

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
  // The exponentials are the hardware's (relative error about 2^-21 for
  // logits within 10 of the maximum, beside sums in 32 bits).
  __device__ __forceinline__ void softmax(float& inv, float& lse) {
    float m = v[0][0];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int u = 0; u < 4; ++u) m = fmaxf(m, v[c][u]);
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
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
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    // a NaN row (the maximum skips NaN) keeps its NaN sum
    const bool empty = none && s == 0.0f;
    inv = empty ? 0.0f : 1.0f / s;
    lse = empty ? 0.0f : mm + logf(s);
  }
};

// The group that holds token t, or the next one: the first g with
// off[g + 1] > t (G: none).
__device__ __forceinline__ int group_at(const int32_t* __restrict__ off, int G, int64_t t) {
  int lo = 0, hi = G;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (off[mid + 1] > t) hi = mid; else lo = mid + 1;
  }
  return lo;
}
// Group boundary, kept inside [0, T] (no offsets: one group of all tokens).
__device__ __forceinline__ int64_t bound(const int32_t* __restrict__ off, int g, int64_t T) {
  if (off == nullptr) return g == 0 ? 0 : T;
  const int64_t v = off[g];
  return v < 0 ? 0 : v < T ? v : T;
}

struct PartSum {
  float z;  // sum of lse^2
  int n;    // valid tokens
};

// Chunk c = tokens [c C, (c + 1) C): the part of each group g that lies in it
// goes to slot c + g (from one part to the next the chunk, the group or both
// move on, so no two parts share a slot).  Per slot: the sum of probabilities
// and the count of every expert, sum of lse^2, valid tokens.
constexpr int PW = 8;  // waves
template <int LPR, int NC>
__global__ __launch_bounds__(64 * PW) void balance_part_kernel(
    const float* __restrict__ logits, const int32_t* __restrict__ idx,
    const int32_t* __restrict__ off, const uint8_t* __restrict__ mask, int64_t T, int E, int k,
    int G, int C, float* __restrict__ part_p, int32_t* __restrict__ part_c,
    PartSum* __restrict__ part_s, int32_t* __restrict__ ticket) {
  constexpr int R = 64 / LPR;             // tokens a wave takes at once
  constexpr int U = NC == 1 ? 4 : NC <= 2 ? 2 : 1;  // and how many times that is in flight
  constexpr int EP = 4 * LPR * NC;
  __shared__ float ps[PW][EP];
  __shared__ int hist[EP];
  __shared__ float zs[PW];
  __shared__ int ns[PW];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l = lane & (LPR - 1), r = lane / LPR;
  const bool vec = (E & 3) == 0;
  for (int g = blockIdx.x * (64 * PW) + threadIdx.x; g < G; g += gridDim.x * (64 * PW)) ticket[g] = 0;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * C, t1 = min(T, t0 + C);
  for (int g = off == nullptr ? 0 : group_at(off, G, t0); g < G; ++g) {
    const int64_t a = max(t0, bound(off, g, T)), b = min(t1, bound(off, g + 1, T));
    if (bound(off, g, T) >= t1) break;
    if (a >= b) continue;
    for (int e = threadIdx.x; e < EP; e += 64 * PW) hist[e] = 0;
    float acc[NC][4] = {};
    float z = 0.0f;
    int n = 0;
    for (int64_t base = a; base < b; base += PW * R * U) {
      Row<LPR, NC> row[U];
      bool ok[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t t = base + (u * PW + w) * R + r;
        ok[u] = t < b && (mask == nullptr || mask[t] != 0);
        const int64_t tc = t < b ? t : b - 1;
        row[u].load(logits + tc * E, E, l, vec);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float inv, lse;
        row[u].softmax(inv, lse);
        if (ok[u]) {
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[c][q] = __builtin_fmaf(row[u].v[c][q], inv, acc[c][q]);
          if (l == 0) {
            z = __builtin_fmaf(lse, lse, z);
            ++n;
          }
        }
      }
    }
    // the wave's R tokens at a time, then its lanes' rows, then the waves
#pragma unroll
    for (int o = LPR; o < 64; o <<= 1) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[c][q] += __shfl_xor(acc[c][q], o, 64);
      z += __shfl_xor(z, o, 64);
      n += __shfl_xor(n, o, 64);
    }
    if (lane < LPR) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
        *reinterpret_cast<float4*>(&ps[w][4 * (l + LPR * c)]) =
            make_float4(acc[c][0], acc[c][1], acc[c][2], acc[c][3]);
    }
    if (lane == 0) {
      zs[w] = z;
      ns[w] = n;
    }
    __syncthreads();  // hist is clear, the sums are there
    const int m = static_cast<int>(b - a) * k;  // at most C k
    for (int i = threadIdx.x; i < m; i += 64 * PW) {
      const int e = idx[a * k + i];
      if (static_cast<unsigned>(e) < static_cast<unsigned>(E) &&
          (mask == nullptr || mask[a + i / k] != 0))
        atomicAdd(&hist[e], 1);
    }
    __syncthreads();
    const int64_t slot = static_cast<int64_t>(blockIdx.x) + g;
    for (int e = threadIdx.x; e < E; e += 64 * PW) {
      float s = ps[0][e];
#pragma unroll
      for (int q = 1; q < PW; ++q) s += ps[q][e];
      part_p[slot * E + e] = s;
      part_c[slot * E + e] = hist[e];
    }
    if (threadIdx.x == 0) {
      PartSum s{zs[0], ns[0]};
      for (int q = 1; q < PW; ++q) {
        s.z += zs[q];
        s.n += ns[q];
      }
      part_s[slot] = s;
    }
    __syncthreads();
  }
}

// Group blockIdx.y, experts 32 blockIdx.x .. + 31: sums over the group's slots,
// eight ranges of slots in parallel, each ascending, then added in order.  The
// last workgroup of a group to finish (by a ticket) adds the groups of 32
// experts in order and forms the losses.
constexpr int RE = 32, RS = 16;
__global__ __launch_bounds__(RE * RS) void balance_reduce_kernel(
    const float* __restrict__ part_p, const int32_t* __restrict__ part_c,
    const PartSum* __restrict__ part_s, const int32_t* __restrict__ off, int64_t T, int E, int k,
    int C, float* __restrict__ balance, float* __restrict__ zloss, int32_t* __restrict__ counts,
    float* __restrict__ prob_sum, int32_t* __restrict__ n_tokens, float* __restrict__ dots,
    int32_t* __restrict__ ticket) {
  __shared__ float fs[RS][RE];
  __shared__ int is[RS][RE];
  __shared__ int is_last;
  const int g = blockIdx.y, EB = gridDim.x;
  const int q = threadIdx.x % RE, sl = threadIdx.x / RE;
  const int e = blockIdx.x * RE + q;
  const int64_t a = bound(off, g, T), b = bound(off, g + 1, T);
  const int64_t s0 = a / C + g, s1 = a < b ? (b - 1) / C + g + 1 : s0;
  const int64_t per = (s1 - s0 + RS - 1) / RS;
  float p = 0.0f;
  int n = 0;
  if (e < E) {
#pragma unroll 4
    for (int64_t s = s0 + sl * per; s < min(s1, s0 + (sl + 1) * per); ++s) {
      p += part_p[s * E + e];
      n += part_c[s * E + e];
    }
  }
  fs[sl][q] = p;
  is[sl][q] = n;
  __syncthreads();
  if (sl == 0) {
    for (int i = 1; i < RS; ++i) {
      p += fs[i][q];
      n += is[i][q];
    }
    if (e < E) {
      counts[static_cast<int64_t>(g) * E + e] = n;
      prob_sum[static_cast<int64_t>(g) * E + e] = p;
    }
    float dot = static_cast<float>(n) * p;
#pragma unroll
    for (int o = 1; o < RE; o <<= 1) dot += __shfl_xor(dot, o, 64);
    if (q == 0) {
      dots[static_cast<int64_t>(g) * EB + blockIdx.x] = dot;
      __threadfence();
      is_last = EB == 1 || atomicAdd(&ticket[g], 1) == EB - 1;
    }
  }
  __syncthreads();
  if (!is_last) return;
  __threadfence();
  // sum of lse^2 and the valid tokens
  float z = 0.0f;
  int nt = 0;
  for (int64_t s = s0 + threadIdx.x; s < s1; s += RE * RS) {
    z += part_s[s].z;
    nt += part_s[s].n;
  }
  z = wave_sum(z);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) nt += __shfl_xor(nt, o, 64);
  if ((threadIdx.x & 63) == 0) {
    fs[0][threadIdx.x >> 6] = z;
    is[0][threadIdx.x >> 6] = nt;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < RE * RS / 64; ++i) {
      z += fs[0][i];
      nt += is[0][i];
    }
    float dot = 0.0f;
    for (int i = 0; i < EB; ++i)
      dot += __hip_atomic_load(&dots[static_cast<int64_t>(g) * EB + i], __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
    const float inv = nt > 0 ? 1.0f / static_cast<float>(nt) : 0.0f;
    balance[g] = static_cast<float>(E) / static_cast<float>(k) * (dot * inv) * inv;
    zloss[g] = z * inv;
    n_tokens[g] = nt;
  }
}

// Logit gradients of BC tokens a workgroup.  Tokens outside every group, masked
// ones and those of a group of no valid tokens get 0 (accumulate: are left).
constexpr int BC = 64;
template <int LPR, int NC>
__global__ __launch_bounds__(256) void balance_bwd_kernel(
    const float* __restrict__ logits, const int32_t* __restrict__ off,
    const uint8_t* __restrict__ mask, const int32_t* __restrict__ counts,
    const int32_t* __restrict__ n_tokens, const float* __restrict__ dbalance,
    const float* __restrict__ dzloss, int64_t T, int E, int k, int G, int accumulate,
    float* __restrict__ dlogits) {
  constexpr int R = 64 / LPR;
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
    float ae[NC][4] = {};
    float fz = 0.0f;
    if (inside) {
      const int n = n_tokens[g];
      const float inv = n > 0 ? 1.0f / static_cast<float>(n) : 0.0f;
      const float fb = dbalance[g] * inv * (static_cast<float>(E) / static_cast<float>(k) * inv);
      fz = 2.0f * dzloss[g] * inv;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int e = 4 * (l + LPR * c) + u;
          ae[c][u] = e < E ? fb * static_cast<float>(counts[static_cast<int64_t>(g) * E + e]) : 0.0f;
        }
    }
    for (int64_t base = at; base < b; base += 4 * R) {
      const int64_t t = base + w * R + r;
      const bool row_ok = t < b;
      const bool ok = row_ok && inside && (mask == nullptr || mask[t] != 0);
      Row<LPR, NC> row;
      row.load(logits + (row_ok ? t : b - 1) * E, E, l, vec);
      float inv, lse;
      row.softmax(inv, lse);
      float s = 0.0f;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          row.v[c][u] *= inv;
          s = __builtin_fmaf(ae[c][u], row.v[c][u], s);
        }
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
      const float add = __builtin_fmaf(fz, lse, -s);
      if (!row_ok || (accumulate && !ok)) continue;
      float* out = dlogits + t * E;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int e = 4 * (l + LPR * c);
        float d[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) d[u] = ok ? row.v[c][u] * (ae[c][u] + add) : 0.0f;
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
          for (int u = 0; u < 4; ++u)
            if (e + u < E) out[e + u] = accumulate ? out[e + u] + d[u] : d[u];
        }
      }
    }
    at = b;
  }
}

// Calls f with the lanes per row and 16-byte pieces per lane that hold E
// experts with the fewest empty lanes.
template <typename F>
hipError_t with_shape(int E, F&& f) {
  auto go = [&](auto L, auto N) { return f(L, N); };
#define MOE_SHAPE(L, N) return go(std::integral_constant<int, L>{}, std::integral_constant<int, N>{})
  const int need = (E + 3) / 4;
  if (need <= 1) MOE_SHAPE(1, 1);
  if (need <= 2) MOE_SHAPE(2, 1);
  if (need <= 4) MOE_SHAPE(4, 1);
  if (need <= 8) MOE_SHAPE(8, 1);
  if (need <= 16) MOE_SHAPE(16, 1);
  if (need <= 32) MOE_SHAPE(32, 1);
  if (need <= 64) MOE_SHAPE(64, 1);
  if (need <= 96) MOE_SHAPE(32, 3);
  if (need <= 128) MOE_SHAPE(64, 2);
  if (need <= 192) MOE_SHAPE(64, 3);
  MOE_SHAPE(64, 4);
#undef MOE_SHAPE
}

// Tokens of a chunk: about one workgroup per compute unit, at least 64 tokens.
int part_chunk(int64_t T) {
  return static_cast<int>(align_up(static_cast<size_t>(std::max<int64_t>(64, ceil_div(T, 256))), 64));
}

}  // namespace

size_t balance_ws_bytes(int64_t T, int E, int G) {
  const size_t slots = static_cast<size_t>(ceil_div(T, part_chunk(T))) + G;
  return 2 * align_up(sizeof(float) * slots * E, 256) + align_up(sizeof(PartSum) * slots, 256) +
         align_up(sizeof(float) * static_cast<size_t>(G) * ceil_div(E, RE), 256) +
         align_up(sizeof(int32_t) * static_cast<size_t>(G), 256);
}

hipError_t launch_balance_fwd(const float* logits, const int32_t* idx, const int32_t* off,
                              const uint8_t* mask, int64_t T, int E, int k, int G, float* balance,
                              float* zloss, int32_t* counts, float* prob_sum, int32_t* n_tokens,
                              void* ws, hipStream_t s) {
  const int C = part_chunk(T);
  const int64_t chunks = ceil_div(T, C);
  const size_t slots = static_cast<size_t>(chunks) + G;
  char* p = static_cast<char*>(ws);
  float* part_p = reinterpret_cast<float*>(p);
  p += align_up(sizeof(float) * slots * E, 256);
  int32_t* part_c = reinterpret_cast<int32_t*>(p);
  p += align_up(sizeof(int32_t) * slots * E, 256);
  PartSum* part_s = reinterpret_cast<PartSum*>(p);
  p += align_up(sizeof(PartSum) * slots, 256);
  float* dots = reinterpret_cast<float*>(p);
  p += align_up(sizeof(float) * static_cast<size_t>(G) * ceil_div(E, RE), 256);
  int32_t* ticket = reinterpret_cast<int32_t*>(p);
  prof_begin(K_BALANCE_PART, s);
  const hipError_t e = with_shape(E, [&](auto L, auto N) {
    balance_part_kernel<L, N><<<static_cast<unsigned>(std::max<int64_t>(1, chunks)), 64 * PW, 0, s>>>(
        logits, idx, off, mask, T, E, k, G, C, part_p, part_c, part_s, ticket);
    return hipGetLastError();
  });
  prof_end(K_BALANCE_PART, s);
  if (e != hipSuccess) return e;
  prof_begin(K_BALANCE_SUM, s);
  balance_reduce_kernel<<<dim3(static_cast<unsigned>(ceil_div(E, RE)), static_cast<unsigned>(G)),
                          RE * RS, 0, s>>>(part_p, part_c, part_s, off, T, E, k, C, balance, zloss,
                                           counts, prob_sum, n_tokens, dots, ticket);
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
    balance_bwd_kernel<L, N><<<static_cast<unsigned>(ceil_div(T, BC)), 256, 0, s>>>(
        logits, off, mask, counts, n_tokens, dbalance, dzloss, T, E, k, G, accumulate, dlogits);
    return hipGetLastError();
  });
  prof_end(K_BALANCE_BWD, s);
  return e;
}

}  // namespace moe
