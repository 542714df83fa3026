// Blockwise vocabulary projection loss (the MoP paper's data-tensor-parallel
// projection, Sec. 3.4 eq. voc-fwd-loss, on one device: P = 1, blocks of the
// vocabulary instead of ranks).  Y = X W_voc is never written anywhere:
//  * forward, per block of `vblock` columns: one bf16 matrix-core product
//    whose epilogue reduces each row's logits to a (max, sum exp(y - max))
//    pair per 64 columns and picks up the target's logit; a one-wave-per-row
//    kernel merges the block's pairs, in column order, into the row's running
//    pair (blocks in order, so the result is a function of the inputs and
//    vblock alone, bit for bit).  The forward walks as many of the caller's
//    blocks at once as its partial pairs fit the workspace for (fwd_span
//    below);
//  * backward, per block: the product is recomputed and its epilogue turns
//    each logit into the logit gradient G = dl ([v == t] - exp(y - lse)),
//    rounded to bf16 (the only per-block buffer, N x vblock bf16); then
//    dX += G W_block^T (fp32, the block's columns cut into K ranges that
//    accumulate into separate fp32 slabs so the product fills the chip) and
//    dW[:, block] = X^T G (bf16, each column written once).
// All products run on the library's grouped GEMM kernel (dense modes).  When
// V is not a multiple of 8 the rows of W and dW are not 16-byte aligned: each
// block of W is first copied into a padded buffer (the product's direct loads
// to LDS want aligned pieces), dW is stored in place.  The same copy takes the
// place of rows so long that a tile's rows lie further apart than a buffer
// descriptor reaches (beyond 34 million columns in the forward, 4 million in
// the backward), and blocks longer than that are cut (reach, below).
//
// Distillation from a teacher's top logits is the same walk with y / tau in
// place of y: the forward's epilogue also picks up the student's logits at the
// teacher's slots, and the backward's is G = dl / tau P exp(y / tau - lse), the
// teacher's probabilities being subtracted at its slots (a few of every
// thousand columns) by a small kernel before the two products.
//
// Sums, exponentials and log-sum-exps are fp32.  G is the one value held in fewer
// bits: rounded to bf16 once (off by 2^-8 of itself at most), as the operand of
// two bf16 matrix products.  Entries round independently and average out in dX
// and dW (their errors against 64 bits, N = 1000, H = 520, V = 32003: 0.0024 of
// their norm; rounding the results alone makes 0.0017), but for the large ones, at
// the teacher's slots, where these are alike: equal dl and probabilities near one
// all round the same way (N = 502, V = 121106, two slots: 0.0029).  With few rows
// such entries are all there is (up to 0.0034), so distillation then holds G in
// two bf16 parts (PARTS_ROWS below).
#include "common.h"

#include <algorithm>

namespace moe {
namespace {

// What the forward of distillation keeps of a teacher: the probability of each
// slot [N][K] and the sum of p log p of each row.
struct DistRows {
  const float* p;
  const float* plogp;
  int K;
  float it;  // 1 / tau
};

// Merge of two (max, sum of exp(y - max)) pairs; an empty pair is (-inf, 0).  A
// sum of NaN stays NaN (its maximum is never -inf).
// The fused add is written out, so that every caller rounds alike.
__device__ __forceinline__ void lse_merge(float& m, float& s, float m2, float s2) {
  const float mm = fmaxf(m, m2);
  if (mm == -__builtin_huge_valf()) return;  // both empty
  s = __builtin_fmaf(s2, __expf(m2 - mm), s * __expf(m - mm));
  m = mm;
}

// W waves per row n: the partial pairs part[n][0..ng) of the caller's blocks
// of per groups each (the last may have fewer).  A block's pairs are merged in
// order (lane l takes groups l, l + 64, ... ascending, then a fixed xor tree
// over the lanes); the blocks' pairs then go into the row's running pair
// (m, s) in order, so the result does not depend on how many blocks a launch
// takes.  A block of fewer than 64 groups takes `sub` lanes of a wave (a power
// of two, per <= sub): the other lanes would hold empty pairs, which merge
// without a trace.  The last launch turns the row's pair into its results:
// lse_n = m_n + log s_n, loss_n = y_{n, t_n} - lse_n.  Bound by latency (loads,
// then up to twelve dependent shuffles and exponentials a block): where one
// wave would come round its 64 / sub blocks often, four waves share a row, 128 /
// sub blocks each at a time (N = 1000, H = 520, V = 32003 in blocks of 4096,
// loss and gradients: 497 us against 500 with one wave a row, and 499 with the
// results in a launch of their own; forward of N = 2048, H = 64, V = 8192 in
// blocks of 512: 20 us, with sub = 64 27, with sub = 8 but four waves 22).
// DIST (distillation): loss_n = sum_s p_s log p_s + sum_s p_s (lse_n - y_{n, s} / tau).
template <int W, bool DIST>
__global__ __launch_bounds__(256) void voc_merge_kernel(const float2* __restrict__ part, int ng,
                                                        int per, int sub, int64_t N,
                                                        float* __restrict__ m,
                                                        float* __restrict__ s, int first, int last,
                                                        const float* __restrict__ yt,
                                                        float* __restrict__ loss,
                                                        float* __restrict__ lse, DistRows q) {
  constexpr int U = W == 1 ? 1 : 2;
  __shared__ float2 blk[W == 1 ? 1 : 64 * U * W];  // a block's pair each
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wv = wave % W;
  const int64_t n = static_cast<int64_t>(blockIdx.x) * (4 / W) + wave / W;
  if (n >= N) return;  // W = 4: the whole workgroup
  const int nsub = 64 / sub, li = lane & (sub - 1), sl = lane / sub;
  const int nb = U * W * nsub;  // blocks at a time
  const float2* row = part + n * ng;
  float rm = 0.0f, rs = 0.0f;
  if (!first) {
    rm = m[n];
    rs = s[n];
  }
  for (int g0 = 0; g0 < ng; g0 += nb * per) {
    float tm[U], ts[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      tm[u] = -__builtin_huge_valf();
      ts[u] = 0.0f;
      const int b = g0 + ((u * W + wv) * nsub + sl) * per, e = b + per < ng ? b + per : ng;
      for (int c = b + li; c < e; c += sub) {
        const float2 p = row[c];
        lse_merge(tm[u], ts[u], p.x, p.y);
      }
    }
    for (int o = 1; o < sub; o <<= 1) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float m2 = __shfl_xor(tm[u], o, 64), s2 = __shfl_xor(ts[u], o, 64);
        // both lanes of a pair compute the same merge in the same operand order
        float a = lane & o ? m2 : tm[u], b = lane & o ? s2 : ts[u];
        lse_merge(a, b, lane & o ? tm[u] : m2, lane & o ? ts[u] : s2);
        tm[u] = a;
        ts[u] = b;
      }
    }
    if constexpr (W == 1) {
      for (int q = 0; q < nsub && g0 + q * per < ng; ++q) {
        const float pm = __shfl(tm[0], q * sub, 64), ps = __shfl(ts[0], q * sub, 64);
        if (first && g0 == 0 && q == 0) {
          rm = pm;
          rs = ps;
        } else {
          lse_merge(rm, rs, pm, ps);
        }
      }
    } else {
      if (li == 0) {
#pragma unroll
        for (int u = 0; u < U; ++u) blk[(u * W + wv) * nsub + sl] = make_float2(tm[u], ts[u]);
      }
      __syncthreads();
      for (int q = 0; q < nb && g0 + q * per < ng; ++q) {
        const float2 p = blk[q];
        if (first && g0 == 0 && q == 0) {
          rm = p.x;
          rs = p.y;
        } else {
          lse_merge(rm, rs, p.x, p.y);
        }
      }
      __syncthreads();
    }
  }
  if constexpr (DIST) {
    if (last) {
      if (wv != 0) return;
      const float l = rm + logf(rs);
      float a = 0.0f;
      for (int j = lane; j < q.K; j += 64) {
        const float p = q.p[n * q.K + j];
        if (p != 0.0f) a = __builtin_fmaf(p, l - yt[n * q.K + j] * q.it, a);
      }
      a = wave_sum(a);
      if (lane == 0) {
        lse[n] = l;
        loss[n] = q.plogp[n] + a;
      }
      return;
    }
  }
  if (lane == 0 && wv == 0) {
    if (last) {
      const float l = rm + logf(rs);
      lse[n] = l;
      loss[n] = yt[n] - l;
    } else {
      m[n] = rm;
      s[n] = rs;
    }
  }
}

// The teacher's probabilities of one row over a wave: lane l holds slots l, l +
// 64, ...  p = 0 where a slot is absent (or its logit -inf); returns their sum,
// and the sum of p log p.
constexpr int DK = MOE_DISTILL_MAX_K / 64;
__device__ __forceinline__ void teacher_row(const Teacher& q, float it, int64_t n, int64_t V, int lane,
                                            int (&id)[DK], float (&p)[DK], float& P, float& plogp) {
  constexpr float NEG = -__builtin_huge_valf();
  float m = NEG;
#pragma unroll
  for (int i = 0; i < DK; ++i) {
    const int j = lane + 64 * i;
    id[i] = j < q.K ? q.ids[n * q.K + j] : -1;
    if (id[i] >= V) id[i] = -1;
    p[i] = id[i] >= 0 ? q.t[n * q.K + j] * it : NEG;
    if (p[i] == -NEG) p[i] = __builtin_nanf("");  // no probability: the row becomes NaN
    m = fmaxf(m, p[i]);
  }
  float shift;
  if (q.tlse != nullptr) {
    shift = q.tlse[n];
  } else {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    const float mm = m == NEG ? 0.0f : m;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < DK; ++i) s += id[i] >= 0 ? expf(p[i] - mm) : 0.0f;
    s = wave_sum(s);
    shift = s == 0.0f ? 0.0f : mm + logf(s);  // s = 0: every p below is 0
  }
  float a = 0.0f, b = 0.0f;
#pragma unroll
  for (int i = 0; i < DK; ++i) {
    const float lp = p[i] - shift;
    p[i] = id[i] >= 0 && p[i] != NEG ? expf(lp) : 0.0f;
    a += p[i];
    if (p[i] != 0.0f) b = __builtin_fmaf(p[i], lp, b);
  }
  P = wave_sum(a);
  plogp = wave_sum(b);
}

// Forward, before the product over columns [b0, b0 + vb): one wave per row.
// first: the teacher's probabilities, their p log p, the slots' ids with -1 for
// absent ones (rows of Kp), and zeros for the absent ones' logits.  Then the
// row's bits, one per 64 of the columns, set where a slot lies in them.
constexpr int DW = 512;  // words of bits in LDS at a time
__global__ __launch_bounds__(256) void distill_prep_kernel(Teacher q, float it, int64_t N, int64_t V,
                                                           int64_t b0, int vb, int hw, int Kp,
                                                           int first, float* __restrict__ p_out,
                                                           float* __restrict__ plogp_out,
                                                           int32_t* __restrict__ ids_out,
                                                           float* __restrict__ yk,
                                                           uint32_t* __restrict__ hits) {
  __shared__ uint32_t bits[4][DW];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t n = static_cast<int64_t>(blockIdx.x) * 4 + w;
  int id[DK];
#pragma unroll
  for (int i = 0; i < DK; ++i) id[i] = -1;
  if (n < N) {
    if (first) {
      float p[DK], P, plogp;
      teacher_row(q, it, n, V, lane, id, p, P, plogp);
#pragma unroll
      for (int i = 0; i < DK; ++i) {
        const int j = lane + 64 * i;
        if (j < q.K) {
          p_out[n * q.K + j] = p[i];
          if (id[i] < 0) yk[n * q.K + j] = 0.0f;
        }
        if (j < Kp) ids_out[n * Kp + j] = id[i];
      }
      if (lane == 0) plogp_out[n] = plogp;
    } else {
#pragma unroll
      for (int i = 0; i < DK; ++i)
        if (lane + 64 * i < Kp) id[i] = ids_out[n * Kp + lane + 64 * i];
    }
  }
  for (int w0 = 0; w0 < hw; w0 += DW) {
    const int nw = hw - w0 < DW ? hw - w0 : DW;
    for (int i = lane; i < nw; i += 64) bits[w][i] = 0u;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < DK; ++i) {
      const int64_t c = id[i] - b0;
      const int64_t g = c >> 6, word = (g >> 5) - w0;
      if (id[i] >= 0 && c >= 0 && c < vb && word >= 0 && word < nw)
        atomicOr(&bits[w][word], 1u << (g & 31));
    }
    __syncthreads();
    if (n < N)
      for (int i = lane; i < nw; i += 64) hits[n * hw + w0 + i] = bits[w][i];
    __syncthreads();
  }
}

// Backward, once: coef_n = dl_n P_n / tau, and of each vocabulary entry that a
// row's slots name the sum of dl_n p_s / tau over them, at the first of them
// (at: its entry; -1 at the others and at absent slots).  x2 (few rows, else
// null): x [N][H] twice, one below the other.
__global__ __launch_bounds__(256) void distill_coef_kernel(Teacher q, float it, int64_t N, int64_t V,
                                                           const float* __restrict__ dloss,
                                                           float* __restrict__ coef,
                                                           float* __restrict__ dp,
                                                           int32_t* __restrict__ at,
                                                           const uint16_t* __restrict__ x, int H,
                                                           uint16_t* __restrict__ x2) {
  const int lane = threadIdx.x & 63;
  const int64_t n = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (n >= N) return;
  if (x2 != nullptr)
    for (int h = 8 * lane; h < H; h += 8 * 64) {
      const uint4 v = *reinterpret_cast<const uint4*>(x + n * H + h);
      *reinterpret_cast<uint4*>(x2 + n * H + h) = v;
      *reinterpret_cast<uint4*>(x2 + (N + n) * H + h) = v;
    }
  int id[DK];
  float p[DK], P, plogp;
  teacher_row(q, it, n, V, lane, id, p, P, plogp);
  const float dl = dloss[n] * it;
  if (lane == 0) coef[n] = dl * P;
  float sum[DK];
  bool first[DK];
#pragma unroll
  for (int i = 0; i < DK; ++i) {
    sum[i] = p[i];
    first[i] = id[i] >= 0;
  }
#pragma unroll
  for (int i2 = 0; i2 < DK; ++i2) {
    const int m = q.K - 64 * i2 < 64 ? q.K - 64 * i2 : 64;
    for (int j = 0; j < m; ++j) {  // slot 64 i2 + j against this lane's
      const int o = __builtin_amdgcn_readlane(id[i2], j);
      const float op = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(p[i2]), j));
#pragma unroll
      for (int i = 0; i < DK; ++i) {
        const bool same = id[i] == o;
        const bool before = i2 < i || (i2 == i && j < lane), after = i2 > i || (i2 == i && j > lane);
        first[i] = first[i] && !(same && before);
        sum[i] += same && after ? op : 0.0f;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < DK; ++i) {
    const int j = lane + 64 * i;
    if (j < q.K) {
      dp[n * q.K + j] = dl * sum[i];
      at[n * q.K + j] = first[i] ? id[i] : -1;
    }
  }
}

// Backward, per block: G at the slots in its columns, from the forward's logits
// there: G = coef exp(y / tau - lse) - dp, one rounding (low: and what it left,
// `low` elements on).  Thread = slot.
__global__ __launch_bounds__(256) void distill_slots_kernel(int K, float it, int64_t N, int64_t b0,
                                                            int vb, const float* __restrict__ coef,
                                                            const float* __restrict__ dp,
                                                            const int32_t* __restrict__ at,
                                                            const float* __restrict__ yk,
                                                            const float* __restrict__ lse,
                                                            uint16_t* __restrict__ G, int64_t gp,
                                                            int64_t low) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= N * K) return;
  const int id = at[i];
  if (id < b0 || id - b0 >= vb) return;
  const int64_t n = i / K;
  const float c = coef[n], a = dp[i];
  const float v = c != 0.0f ? __builtin_fmaf(c, __expf(__builtin_fmaf(yk[i], it, -lse[n])), -a) : -a;
  uint16_t* const to = G + n * gp + (id - b0);
  *to = static_cast<uint16_t>(f32_to_bf16_bits(v));
  if (low != 0) to[low] = static_cast<uint16_t>(f32_to_bf16_bits(v - bf16_to_f32(*to)));
}

// Workgroups of 256 threads for n items of a kernel that steps over what is
// beyond its grid: a launch holds less than 2^32 threads, and 2^16 workgroups
// fill the chip many times over.
unsigned groups_for(int64_t n) {
  return static_cast<unsigned>(std::min<int64_t>(ceil_div(n, 256), 1 << 16));
}

// dx[i] = bf16(sum over slabs b ascending of dxa[b][i]), 8 values per thread
// and step (n = N H is a multiple of 8), eight slabs' loads in flight at once
__global__ __launch_bounds__(256) void voc_dx_sum_kernel(const float* __restrict__ dxa, int slabs,
                                                         int64_t n, uint16_t* __restrict__ dx) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * 256 * 8;
  for (int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8; i < n; i += step) {
    float v[8];
    {
      const float4 a = *reinterpret_cast<const float4*>(dxa + i);
      const float4 b = *reinterpret_cast<const float4*>(dxa + i + 4);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
#pragma unroll 8
    for (int sl = 1; sl < slabs; ++sl) {
      const float* p = dxa + static_cast<int64_t>(sl) * n + i;
      const float4 a = *reinterpret_cast<const float4*>(p);
      const float4 b = *reinterpret_cast<const float4*>(p + 4);
      v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z;
      v[7] += b.w;
    }
    *reinterpret_cast<uint4*>(dx + i) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                                   pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  }
}

// wst[h][c] = c < vb ? w[h][v0 + c] : 0 for c < vbp (padded copy of a block),
// eight columns a thread and step, read together whatever their alignment (H =
// 520, V = 32003: 11 us; two bytes at a time 22)
__global__ __launch_bounds__(256) void voc_stage_kernel(const uint16_t* __restrict__ w, int64_t V,
                                                        int64_t v0, int vb, int vbp, int H,
                                                        uint16_t* __restrict__ wst) {
  const int per = vbp / 8;
  const int64_t n = static_cast<int64_t>(H) * per;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t h = i / per;
    const int c = static_cast<int>(i - h * per) * 8;
    const uint16_t* src = w + h * V + v0 + c;
    uint32_t p[4];
    if (c + 8 <= vb) {
      __builtin_memcpy(p, src, 16);  // one load, of any alignment
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t lo = c + 2 * q < vb ? src[2 * q] : 0u;
        const uint32_t hi = c + 2 * q + 1 < vb ? src[2 * q + 1] : 0u;
        p[q] = lo | (hi << 16);
      }
    }
    *reinterpret_cast<uint4*>(wst + i * 8) = make_uint4(p[0], p[1], p[2], p[3]);
  }
}

hipError_t stage(const uint16_t* w, int64_t V, int64_t v0, int vb, int vbp, int H, uint16_t* wst,
                 hipStream_t s) {
  const int64_t n = static_cast<int64_t>(H) * (vbp / 8);
  voc_stage_kernel<<<groups_for(n), 256, 0, s>>>(w, V, v0, vb, vbp, H, wst);
  return hipGetLastError();
}

// n, a multiple of 8, zeros at a 16-byte aligned p, eight a thread and step
__global__ __launch_bounds__(256) void voc_zero_bf16_kernel(uint16_t* __restrict__ p, int64_t n) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * 256 * 8;
  for (int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8; i < n; i += step)
    *reinterpret_cast<uint4*>(p + i) = make_uint4(0u, 0u, 0u, 0u);
}

// The products address a tile's rows of an operand by 32-bit offsets from the
// first, within the 2^31 - 16 bytes of a buffer descriptor: true if `rows`
// rows of `pitch` elements, the last read up to element `tail`, fit.  Rows per
// operand: 32 (one half step) where the contraction index runs over rows (W in
// the logits, G in dW), 256 (a tile) where it runs along them (G and W in dX).
constexpr int64_t REACH = 0x7ffffff0;
bool reach(int64_t rows, int64_t pitch, int64_t tail) {
  return 2 * ((rows - 1) * pitch + tail) <= REACH;
}
// the longest pitch (a multiple of 64) whose `rows` rows fit
int64_t max_pitch(int64_t rows) { return REACH / (2 * rows) / 64 * 64; }

// W read through a padded copy of a block?
bool staged_fwd(int H, int64_t V) {
  return (V % 8) != 0 || !reach(std::min(H, 32), V, 128);
}
bool staged_bwd(int H, int64_t V, int64_t vb) {
  return staged_fwd(H, V) || !reach(std::min(H, 256), V, std::min(vb, V));
}
// The caller's block, cut where the copy (forward) or G and the copy
// (backward) would have rows out of reach.
int64_t fwd_block(int H, int64_t V, int64_t vblock) {
  const int64_t most = max_pitch(std::min(H, 32));
  return staged_fwd(H, V) && std::min(vblock, V) > most ? most : vblock;
}
// The block that the forward walks: the caller's, less what is beyond a whole
// number of groups of 64 columns.  A block that ended inside a group could not
// be part of a longer product (its columns would fall into other groups, and
// the pairs be other sums), and had to be a launch of its own: N = 500, H =
// 520, V = 32000 in blocks of 1000 took 458 us in 32 launches, 35 in one.
int64_t fwd_step(int H, int64_t V, int64_t vblock) {
  const int64_t b = fwd_block(H, V, vblock);
  return b < V && b > 64 ? b / 64 * 64 : b;
}
int64_t bwd_block(int64_t N, int H, int64_t V, int64_t vblock) {
  const int64_t rows = std::max<int64_t>(N, staged_bwd(H, V, vblock) ? H : 1);
  const int64_t most = max_pitch(std::min<int64_t>(rows, 256));
  return std::min(vblock, V) > most ? most : vblock;
}

// K ranges of the dX product: enough (row tile x column tile x range) work
// items for about two per compute unit of a 256-CU device, each range at
// least 512 columns (a multiple of 64; distillation's about 512).  At most 8,
// and more only of distillation (the loss keeps the order of its sums) with few
// tokens: as many as stay on the 128-row tile, whose four times as many items
// then fill the chip, and whose partial sums are fewer bytes than W (N = 4, H =
// 616, V = 70554: 20 us, in 8 ranges 87; twice as many ranges, on the 256-row tile,
// with N = 1, H = 3792, V = 77664 155 us against 105).
int64_t dx_kspan(int64_t N, int H, int64_t V, int64_t vblock, int K) {
  if (K > 0) vblock = std::min(vblock, V);
  const int64_t tiles = std::max<int64_t>(1, ceil_div(N, 256) * ceil_div(H, 256));
  int64_t S = std::min<int64_t>(8, std::max<int64_t>(1, ceil_div(512, tiles)));
  if (K > 0)
    S = std::max<int64_t>(S, std::min<int64_t>(2 * 256 / 3 / tiles, vblock / (4 * std::max<int64_t>(N, 1))));
  S = std::max<int64_t>(1, std::min<int64_t>(S, K > 0 ? ceil_div(vblock, 512) : vblock / 512));
  return align_up(static_cast<size_t>(ceil_div(vblock, S)), 64);
}

}  // namespace

namespace {
// Words of 32 bits that a row's columns take, one bit per 64 of them.
int hit_words(int64_t vb) { return static_cast<int>(ceil_div(ceil_div(vb, 64), 32)); }
int padded_slots(int K) { return static_cast<int>(align_up(static_cast<size_t>(K), 4)); }

// Up to how many rows distillation's G is the sum of two bf16 parts (2^-16 of an
// entry off) held as 2 N rows: dX is a product of 2 N rows whose halves are added
// with the K ranges' partial sums, dW one over 2 N rows, x twice.  Error of dx and
// dw against 64 bits over that of rounding the results alone, V = 8000 and 20001,
// one part, two parts: N = 1 ... 5 up to 1.99, 1.00; 16 1.53, 1.00; 64 1.47, 1.00;
// 256 1.39.  Forward and backward, H = 1024, V = 50000: N = 64 151 and 178 us; 128
// 173 and 220; 256 206 and 293 (H = 4096, V = 151669 unaligned, N = 64: 2341 and
// 2484: with so few rows most of it is W's).
constexpr int64_t PARTS_ROWS = 64;
int64_t grad_rows(int64_t N, int K) { return K > 0 && N <= PARTS_ROWS ? 2 * N : N; }

// Distillation's backward takes as many of the caller's blocks together as
// keep the logit gradients within 64 MiB, and the copy of W's columns, where
// there is one, within 256 (few rows would otherwise take a copy of all of W,
// whatever the caller's block): a block of its own four launches each costs
// more than it saves where it is small (forward and backward of N = 1000, H =
// 520, V = 32003 in blocks of 4096, 20 slots: 523 us block by block, 300
// together; N = 256, H = 128, V = 1000 in blocks of 256 127 us against 55).
// Copies of at most 64, 128 and 256 MiB and of all of W, N = 64, H = 4096, V =
// 151669 in blocks of 8192: 3549, 2765, 2333 and 2310 us; N = 1, H = 3792, V =
// 77663 in blocks of 304: 1600, 1195, 1194 and 1033.
int64_t together(int64_t rows, int H, int64_t V, int64_t vblock) {
  if (vblock >= V) return vblock;
  constexpr int64_t grad = int64_t{64} << 20, copy = int64_t{256} << 20;
  int64_t m = grad / (2 * std::max<int64_t>(1, rows)) / vblock;
  if (staged_bwd(H, V, m * vblock)) m = std::min(m, copy / (2 * int64_t{H}) / vblock);
  return m > 1 ? vblock * std::min(m, ceil_div(V, vblock)) : vblock;
}

// Workspace of a forward that takes `span` columns at once; K slots of a
// teacher per row (0: the plain loss).
size_t fwd_bytes(int64_t N, int H, int64_t V, int64_t span, int K) {
  const int64_t vb = std::min(span, V);
  const size_t n = static_cast<size_t>(N);
  size_t b = align_up(sizeof(float) * 2 * n * ceil_div(vb, 64), 256);  // pairs
  b += 3 * align_up(sizeof(float) * n, 256);  // running max, sum; target logit (sum of p log p)
  if (K > 0)
    b += align_up(sizeof(float) * n * K, 256) + align_up(sizeof(int32_t) * n * padded_slots(K), 256) +
         align_up(sizeof(uint32_t) * n * hit_words(vb), 256);
  if (staged_fwd(H, V))
    b += align_up(sizeof(uint16_t) * static_cast<size_t>(H) * align_up(vb, 8), 256);
  return b + 256;
}
size_t bwd_bytes(int64_t N, int H, int64_t V, int64_t vblock, int K) {
  const int64_t rows = grad_rows(N, K);
  if (K > 0) vblock = together(rows, H, V, vblock);
  vblock = bwd_block(rows, H, V, vblock);
  const int64_t vb = std::min(vblock, V);
  const int64_t vbp = align_up(vb, 8);
  const int64_t slabs = ceil_div(vb, dx_kspan(rows, H, V, vblock, K));
  size_t b = align_up(sizeof(uint16_t) * static_cast<size_t>(rows) * vbp, 256);         // G
  b += align_up(sizeof(float) * static_cast<size_t>(slabs) * rows * H, 256);             // dX slabs
  if (staged_bwd(H, V, vblock))
    b += align_up(sizeof(uint16_t) * static_cast<size_t>(H) * vbp, 256);  // W
  if (K > 0)
    b += align_up(sizeof(float) * static_cast<size_t>(N), 256) +
         2 * align_up(sizeof(float) * static_cast<size_t>(N) * K, 256);  // coef; dl p, entries
  if (rows > N) b += align_up(sizeof(uint16_t) * static_cast<size_t>(rows) * H, 256);  // x twice
  return b + 256;
}
size_t fwd_least(int64_t N, int H, int64_t V, int64_t vblock, int K) {
  return fwd_bytes(N, H, V, fwd_block(H, V, vblock), K);
}
// Columns the forward takes at once: the largest multiple of vblock whose
// partial pairs (and staged copy of W) fit the workspace that
// moe_vocab_loss_workspace_bytes() asks for, which the backward's buffers
// set.  One product of many tiles instead of one per block: fewer launches
// and partly filled last rounds (N = 1000, H = 520, V = 32003 in blocks of
// 4096: 8 products and merges become 2; N = 4096, H = 2048, V = 200000: 13
// become 1).  Blocks of fewer than 64 columns stay alone.  A copy of W stays
// within reach.
int64_t fwd_span(int64_t N, int H, int64_t V, int64_t vblock, int K) {
  const size_t room = std::max(fwd_least(N, H, V, vblock, K), bwd_bytes(N, H, V, vblock, K));
  vblock = fwd_step(H, V, vblock);
  if (vblock % 64 != 0) return vblock;
  int64_t most = std::min<int64_t>(ceil_div(V, vblock), ((int64_t{1} << 40) - 1) / (N * vblock));
  if (staged_fwd(H, V))
    most = std::min(most, max_pitch(std::min(H, 32)) / vblock);
  int64_t lo = 1, hi = std::max<int64_t>(1, most);  // the largest m in [lo, hi] that fits
  while (lo < hi) {
    const int64_t mid = (lo + hi + 1) / 2;
    if (fwd_bytes(N, H, V, mid * vblock, K) <= room) lo = mid; else hi = mid - 1;
  }
  return lo * vblock;
}
}  // namespace

size_t vocab_fwd_ws_bytes(int64_t N, int H, int64_t V, int64_t vblock) {
  return fwd_least(N, H, V, vblock, 0);
}
size_t vocab_bwd_ws_bytes(int64_t N, int H, int64_t V, int64_t vblock) {
  return bwd_bytes(N, H, V, vblock, 0);
}
size_t distill_fwd_ws_bytes(int64_t N, int H, int64_t V, int64_t vblock, int K) {
  return fwd_least(N, H, V, vblock, K);
}
size_t distill_bwd_ws_bytes(int64_t N, int H, int64_t V, int64_t vblock, int K) {
  return bwd_bytes(N, H, V, vblock, K);
}

namespace {
// f(first, rows) over the N rows in pieces that a launch of a wave a row holds
// (less than 2^32 threads).
template <typename F>
void by_rows(int64_t N, F&& f) {
  constexpr int64_t most = int64_t{1} << 25;
  for (int64_t n0 = 0; n0 < N; n0 += most) f(n0, std::min(most, N - n0));
}
// The teacher of the rows from n0 on.
Teacher from_row(Teacher q, int64_t n0) {
  q.ids += n0 * q.K;
  q.t += n0 * q.K;
  if (q.tlse != nullptr) q.tlse += n0;
  return q;
}

// The forward of either loss: against targets, or a teacher (q, yk).
hipError_t run_fwd(const uint16_t* x, const uint16_t* w, const int32_t* target, const Teacher* q,
                   int64_t N, int H, int64_t V, int64_t vblock, float* loss, float* lse, float* yk,
                   void* ws, size_t ws_bytes, hipStream_t s) {
  if (N == 0) return hipSuccess;
  const int K = q != nullptr ? q->K : 0;
  // a caller with room for the forward alone gets its blocks one by one
  const int64_t span = ws_bytes >= bwd_bytes(N, H, V, vblock, K) ? fwd_span(N, H, V, vblock, K)
                                                                 : fwd_step(H, V, vblock);
  const int64_t vbmax = std::min(span, V);
  // groups of 64 columns per block
  const int per = static_cast<int>(ceil_div(std::min(fwd_step(H, V, vblock), V), 64));
  int sub = 1;
  while (sub < 64 && sub < per) sub *= 2;
  char* p = static_cast<char*>(ws);
  float* part = reinterpret_cast<float*>(p);
  p += align_up(sizeof(float) * 2 * static_cast<size_t>(N) * ceil_div(vbmax, 64), 256);
  float* m = reinterpret_cast<float*>(p);
  p += align_up(sizeof(float) * static_cast<size_t>(N), 256);
  float* sm = reinterpret_cast<float*>(p);
  p += align_up(sizeof(float) * static_cast<size_t>(N), 256);
  float* yt = reinterpret_cast<float*>(p);
  p += align_up(sizeof(float) * static_cast<size_t>(N), 256);
  DistRows rows{};
  float* prob = nullptr;
  int32_t* ids = nullptr;
  uint32_t* hits = nullptr;
  const int Kp = padded_slots(K);
  if (K > 0) {
    prob = reinterpret_cast<float*>(p);
    p += align_up(sizeof(float) * static_cast<size_t>(N) * K, 256);
    ids = reinterpret_cast<int32_t*>(p);
    p += align_up(sizeof(int32_t) * static_cast<size_t>(N) * Kp, 256);
    hits = reinterpret_cast<uint32_t*>(p);
    p += align_up(sizeof(uint32_t) * static_cast<size_t>(N) * hit_words(vbmax), 256);
    rows = DistRows{prob, yt, K, 1.0f / q->tau};
  }
  uint16_t* wst = staged_fwd(H, V) ? reinterpret_cast<uint16_t*>(p) : nullptr;
  const int n = static_cast<int>(N);
  for (int64_t b0 = 0; b0 < V; b0 += span) {
    const int vb = static_cast<int>(std::min<int64_t>(span, V - b0));
    const uint16_t* wb = w;
    int64_t ldw = V, bc0 = b0;
    if (wst != nullptr) {
      const int vbp = static_cast<int>(align_up(vb, 8));
      if (hipError_t e = stage(w, V, b0, vb, vbp, H, wst, s); e != hipSuccess) return e;
      wb = wst;
      ldw = vbp;
      bc0 = 0;
    }
    const int first = b0 == 0, last = b0 + span >= V;
    if (K > 0) {
      const int hw = hit_words(vb);
      prof_begin(K_VOC_TEACHER, s);
      by_rows(N, [&](int64_t n0, int64_t nr) {
        distill_prep_kernel<<<static_cast<unsigned>(ceil_div(nr, 4)), 256, 0, s>>>(
            from_row(*q, n0), rows.it, nr, V, b0, vb, hw, Kp, first, prob + n0 * K, yt + n0, ids + n0 * Kp,
            yk + n0 * K, hits + n0 * hw);
      });
      prof_end(K_VOC_TEACHER, s);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      if (hipError_t e = launch_distill_logits_mfma(x, wb, ldw, bc0, b0, n, H, vb, rows.it, hits, hw,
                                                    ids, K, Kp, part, yk, s);
          e != hipSuccess)
        return e;
    } else if (hipError_t e =
                   launch_vocab_logits_mfma(x, wb, ldw, bc0, b0, n, H, vb, target, part, yt, s);
               e != hipSuccess) {
      return e;
    }
    prof_begin(K_VOC_LSE, s);
    const int ng = static_cast<int>(ceil_div(vb, 64));
    const float2* pairs = reinterpret_cast<const float2*>(part);
    const int64_t rounds = ceil_div(ceil_div(ng, per), 64 / sub);  // of one wave a row
    auto merge = [&](auto DIST) {
      if (rounds <= (sub < 64 ? 4 : 1) || N > (int64_t{1} << 23))  // or rows enough
        by_rows(N, [&](int64_t n0, int64_t nr) {
          voc_merge_kernel<1, DIST><<<static_cast<unsigned>(ceil_div(nr, 4)), 256, 0, s>>>(
              pairs + n0 * ng, ng, per, sub, nr, m + n0, sm + n0, first, last,
              DIST ? yk + n0 * K : yt + n0, loss + n0, lse + n0,
              DistRows{rows.p + n0 * K, rows.plogp + n0, K, rows.it});
        });
      else
        voc_merge_kernel<4, DIST><<<static_cast<unsigned>(N), 256, 0, s>>>(
            pairs, ng, per, sub, N, m, sm, first, last, DIST ? yk : yt, loss, lse, rows);
    };
    if (K > 0) merge(std::true_type{});
    else merge(std::false_type{});
    prof_end(K_VOC_LSE, s);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t run_bwd(const uint16_t* x, const uint16_t* w, const int32_t* target, const Teacher* q,
                   const float* lse, const float* yk, const float* dloss, int64_t N, int H,
                   int64_t V, int64_t vblock, uint16_t* dx, uint16_t* dw, void* ws, hipStream_t s) {
  if (N == 0) {  // no tokens: the weight gradient is exact zeros (dx is empty)
    const int64_t nw = static_cast<int64_t>(H) * V;  // H is a multiple of 8
    voc_zero_bf16_kernel<<<groups_for(nw / 8), 256, 0, s>>>(dw, nw);
    return hipGetLastError();
  }
  const int64_t rows = grad_rows(N, q != nullptr ? q->K : 0);  // of G
  if (q != nullptr) vblock = together(rows, H, V, vblock);
  vblock = bwd_block(rows, H, V, vblock);
  const int64_t vbmax = std::min(vblock, V);
  const int64_t vbpmax = align_up(vbmax, 8);
  // a range longer than the block is the block (vblock itself may exceed an int)
  const int kspan = static_cast<int>(
      std::min<int64_t>(dx_kspan(rows, H, V, vblock, q != nullptr ? q->K : 0),
                        static_cast<int64_t>(align_up(vbmax, 64))));
  const int slabs = static_cast<int>(ceil_div(vbmax, kspan));  // the first block fills them all
  char* p = static_cast<char*>(ws);
  uint16_t* G = reinterpret_cast<uint16_t*>(p);
  p += align_up(sizeof(uint16_t) * static_cast<size_t>(rows) * vbpmax, 256);
  float* dxa = reinterpret_cast<float*>(p);
  p += align_up(sizeof(float) * static_cast<size_t>(slabs) * rows * H, 256);
  uint16_t* wst = nullptr;
  if (staged_bwd(H, V, vblock)) {
    wst = reinterpret_cast<uint16_t*>(p);
    p += align_up(sizeof(uint16_t) * static_cast<size_t>(H) * vbpmax, 256);
  }
  float *coef = nullptr, *dp = nullptr;
  int32_t* at = nullptr;
  const uint16_t* xg = x;  // x of G's rows
  const float it = q != nullptr ? 1.0f / q->tau : 1.0f;
  if (q != nullptr) {
    coef = reinterpret_cast<float*>(p);
    p += align_up(sizeof(float) * static_cast<size_t>(N), 256);
    dp = reinterpret_cast<float*>(p);
    p += align_up(sizeof(float) * static_cast<size_t>(N) * q->K, 256);
    at = reinterpret_cast<int32_t*>(p);
    p += align_up(sizeof(int32_t) * static_cast<size_t>(N) * q->K, 256);
    uint16_t* const x2 = rows > N ? reinterpret_cast<uint16_t*>(p) : nullptr;
    prof_begin(K_VOC_TEACHER, s);
    by_rows(N, [&](int64_t n0, int64_t nr) {
      distill_coef_kernel<<<static_cast<unsigned>(ceil_div(nr, 4)), 256, 0, s>>>(
          from_row(*q, n0), it, nr, V, dloss + n0, coef + n0, dp + n0 * q->K, at + n0 * q->K, x, H, x2);
    });
    if (x2 != nullptr) xg = x2;
    prof_end(K_VOC_TEACHER, s);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  const int n = static_cast<int>(N), nr = static_cast<int>(rows);
  for (int64_t b0 = 0; b0 < V; b0 += vblock) {
    const int vb = static_cast<int>(std::min<int64_t>(vblock, V - b0));
    const int64_t gp = align_up(vb, 8), low = (rows - N) * gp;
    const uint16_t* wb = w;
    int64_t ldw = V, bc0 = b0;
    if (wst != nullptr) {
      if (hipError_t e = stage(w, V, b0, vb, static_cast<int>(gp), H, wst, s); e != hipSuccess)
        return e;
      wb = wst;
      ldw = gp;
      bc0 = 0;
    }
    if (q != nullptr) {
      if (hipError_t e = launch_distill_grad_mfma(x, wb, ldw, bc0, n, H, vb, it, lse, coef, G, gp, low,
                                                      s);
          e != hipSuccess)
        return e;
      prof_begin(K_VOC_TEACHER, s);
      distill_slots_kernel<<<static_cast<unsigned>(ceil_div(N * q->K, 256)), 256, 0, s>>>(
          q->K, it, N, b0, vb, coef, dp, at, yk, lse, G, gp, low);
      prof_end(K_VOC_TEACHER, s);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    } else if (hipError_t e = launch_vocab_grad_mfma(x, wb, ldw, bc0, b0, n, H, vb, target, lse,
                                                     dloss, G, gp, s);
               e != hipSuccess) {
      return e;
    }
    if (hipError_t e = launch_vocab_dx_mfma(G, gp, wb, ldw, bc0, nr, H, vb, kspan, b0 == 0, dxa, s);
        e != hipSuccess)
      return e;
    if (hipError_t e = launch_vocab_dw_mfma(xg, G, gp, nr, H, vb, dw, V, b0, s); e != hipSuccess)
      return e;
  }
  const int64_t nx = N * H;  // (G's parts are slabs of their own)
  voc_dx_sum_kernel<<<groups_for(nx / 8), 256, 0, s>>>(dxa, slabs * static_cast<int>(rows / N), nx, dx);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_vocab_fwd(const uint16_t* x, const uint16_t* w, const int32_t* target,
                            int64_t N, int H, int64_t V, int64_t vblock, float* loss, float* lse,
                            void* ws, size_t ws_bytes, hipStream_t s) {
  return run_fwd(x, w, target, nullptr, N, H, V, vblock, loss, lse, nullptr, ws, ws_bytes, s);
}
hipError_t launch_vocab_bwd(const uint16_t* x, const uint16_t* w, const int32_t* target,
                            const float* lse, const float* dloss, int64_t N, int H, int64_t V,
                            int64_t vblock, uint16_t* dx, uint16_t* dw, void* ws, hipStream_t s) {
  return run_bwd(x, w, target, nullptr, lse, nullptr, dloss, N, H, V, vblock, dx, dw, ws, s);
}
hipError_t launch_distill_fwd(const uint16_t* x, const uint16_t* w, const Teacher& q, int64_t N,
                              int H, int64_t V, int64_t vblock, float* loss, float* lse, float* yk,
                              void* ws, size_t ws_bytes, hipStream_t s) {
  return run_fwd(x, w, nullptr, &q, N, H, V, vblock, loss, lse, yk, ws, ws_bytes, s);
}
hipError_t launch_distill_bwd(const uint16_t* x, const uint16_t* w, const Teacher& q,
                              const float* lse, const float* yk, const float* dloss, int64_t N,
                              int H, int64_t V, int64_t vblock, uint16_t* dx, uint16_t* dw,
                              void* ws, hipStream_t s) {
  return run_bwd(x, w, nullptr, &q, lse, yk, dloss, N, H, V, vblock, dx, dw, ws, s);
}

}  // namespace moe
