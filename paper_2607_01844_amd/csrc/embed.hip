// Embedding of tokens and its weight gradient (gfx950).
//   y[t] = bf16(scale W[ids[t] - begin]),   0 where that is no row of this rank;
//   dW[v] = bf16(scale sum of dy[t] over t with ids[t] - begin = v), t ascending.
// The gradient sorts the tokens by row (stable, so that sums have one order), then
// cuts the sorted list into pieces of equal length, so that a frequent word costs
// no wave more than a rare one: a run of one row inside a piece is summed in
// registers and written; one that passes a piece's end leaves fp32 partial sums,
// which are joined in order.  Rows without tokens are written as zeros by
// workgroups that look them up in the sorted list.  Both directions are bound by
// the HBM stream of their rows, the gradient mostly by writing dW.
#include <algorithm>

#include "common.h"

namespace moe {
namespace {

constexpr int SORT_W = 16;        // waves of a sorting workgroup
constexpr int SORT_SMALL = 8192;  // tokens that one workgroup sorts
constexpr int SORT_BITS = 9;      // widest digit
constexpr int SORT_BLOCKS = 64;   // workgroups of a sorting pass, up to 2^20 tokens
constexpr int ZERO_ROWS = 32;     // rows looked up by a workgroup

__device__ __forceinline__ void unpack8(const uint4& v, float* f) {
  f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x);
  f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
  f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z);
  f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
}
__device__ __forceinline__ uint4 pack8(const float* f) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                    pack_bf16x2(f[6], f[7]));
}

// A token's row of this rank, or `rows` (none).
__device__ __forceinline__ uint32_t row_of(int32_t id, int64_t begin, int64_t rows) {
  const int64_t v = id - begin;
  return static_cast<uint32_t>(v >= 0 && v < rows ? v : rows);
}

// 2^s lanes a token, 8 columns a lane and step.
__global__ __launch_bounds__(256) void embed_fwd_kernel(const int32_t* __restrict__ ids,
                                                        const uint16_t* __restrict__ w, int64_t N,
                                                        int H, int64_t begin, int64_t rows,
                                                        float scale, int s,
                                                        uint16_t* __restrict__ y) {
  const int nch = H >> 3, l = threadIdx.x & ((1 << s) - 1), lanes = 1 << s;
  const int teams = 256 >> s;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * teams + (threadIdx.x >> s); t < N;
       t += static_cast<int64_t>(gridDim.x) * teams) {
    const uint32_t row = row_of(ids[t], begin, rows);
    const bool there = row < rows;
    const uint4* src = reinterpret_cast<const uint4*>(w + static_cast<int64_t>(there ? row : 0) * H);
    uint4* dst = reinterpret_cast<uint4*>(y + t * H);
    constexpr int U = 4;
    for (int c0 = l; c0 < nch; c0 += lanes * U) {
      uint4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        v[u] = make_uint4(0, 0, 0, 0);
        if (there && c0 + u * lanes < nch) v[u] = src[c0 + u * lanes];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float f[8];
        unpack8(v[u], f);
#pragma unroll
        for (int q = 0; q < 8; ++q) f[q] *= scale;
        // an absent row is 0, whatever the scale is
        if (c0 + u * lanes < nch) dst[c0 + u * lanes] = there ? pack8(f) : make_uint4(0, 0, 0, 0);
      }
    }
  }
}

// ------------------------------------------------------------------ sorting
// The lanes of a wave whose digit (nbits of it) equals this one's.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, int nbits, bool in) {
  uint64_t same = __ballot(in);
  for (int b = 0; b < nbits; ++b) {
    const bool bit = (digit >> b) & 1;
    const uint64_t bal = __ballot(bit);
    same &= bit ? bal : ~bal;
  }
  return same;
}
__device__ __forceinline__ int lower_lanes(uint64_t m, int lane) {
  return __popcll(m & (lane == 0 ? 0ull : (~0ull >> (64 - lane))));
}

// Exclusive sums over `bins` <= 512 values, one a thread of the workgroup's first
// `bins` (v = 0 beyond): every thread calls it.
__device__ __forceinline__ int scan_bins(int v, int* wsum) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(incl, o, 64);
    if (lane >= o) incl += y;
  }
  if (lane == 63) wsum[w] = incl;
  __syncthreads();
  int base = 0;
  for (int i = 0; i < w; ++i) base += wsum[i];
  return base + incl - v;
}

// Up to SORT_SMALL tokens in one workgroup: every pass ranks the tokens of each
// wave's slice in order, and places them through LDS.
__global__ __launch_bounds__(64 * SORT_W) void embed_sort_small_kernel(
    const int32_t* __restrict__ ids, int N, int64_t begin, int64_t rows, int passes, int nbits,
    uint32_t* __restrict__ key, int32_t* __restrict__ tok) {
  constexpr int R = SORT_SMALL / (64 * SORT_W);
  __shared__ int cnt[SORT_W << SORT_BITS];
  __shared__ int wsum[SORT_W];
  __shared__ uint64_t ent[SORT_SMALL];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, bins = 1 << nbits;
  const int per = (N + 64 * SORT_W - 1) / (64 * SORT_W);
  const int base = w * per * 64;
  uint64_t e[R];
  int rank[R];
#pragma unroll
  for (int it = 0; it < R; ++it) {
    const int a = base + it * 64 + lane;
    e[it] = 0;
    if (it < per && a < N)
      e[it] = static_cast<uint64_t>(row_of(ids[a], begin, rows)) << 32 | static_cast<uint32_t>(a);
  }
  int* mine = cnt + w * bins;
  for (int p = 0; p < passes; ++p) {
    for (int i = tid; i < SORT_W * bins; i += 64 * SORT_W) cnt[i] = 0;
    __syncthreads();
#pragma unroll
    for (int it = 0; it < R; ++it) {
      if (it < per) {
        const bool in = base + it * 64 + lane < N;
        const uint32_t dg = static_cast<uint32_t>(e[it] >> (32 + p * nbits)) & (bins - 1);
        const uint64_t same = same_digit(dg, nbits, in);
        if (in) {
          const int prev = mine[dg];
          rank[it] = prev + lower_lanes(same, lane);
          if ((same >> lane) == 1ull) mine[dg] = prev + __popcll(same);
        }
        // the next step's lanes read what this step's wrote
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
    }
    __syncthreads();
    int run = 0;
    if (tid < bins)
      for (int u = 0; u < SORT_W; ++u) {
        const int c = cnt[u * bins + tid];
        cnt[u * bins + tid] = run;
        run += c;
      }
    const int first = scan_bins(tid < bins ? run : 0, wsum);
    if (tid < bins)
      for (int u = 0; u < SORT_W; ++u) cnt[u * bins + tid] += first;
    __syncthreads();
#pragma unroll
    for (int it = 0; it < R; ++it)
      if (it < per && base + it * 64 + lane < N) {
        const uint32_t dg = static_cast<uint32_t>(e[it] >> (32 + p * nbits)) & (bins - 1);
        ent[mine[dg] + rank[it]] = e[it];
      }
    __syncthreads();
#pragma unroll
    for (int it = 0; it < R; ++it) {
      const int a = base + it * 64 + lane;
      if (it < per && a < N) e[it] = ent[a];
    }
  }
#pragma unroll
  for (int it = 0; it < R; ++it) {
    const int a = base + it * 64 + lane;
    if (it < per && a < N) {
      key[a] = static_cast<uint32_t>(e[it] >> 32);
      tok[a] = static_cast<int32_t>(e[it]);
    }
  }
}

// More tokens: a pass is two launches of the same blocks.  This one counts the
// digits of every block's tokens; FIRST: keys come from the ids.
template <bool FIRST>
__global__ __launch_bounds__(1024) void embed_count_kernel(
    const int32_t* __restrict__ ids, const uint32_t* __restrict__ key, int64_t N, int64_t chunk,
    int64_t begin, int64_t rows, int shift, int nbits, int32_t* __restrict__ count) {
  __shared__ int cnt[1 << SORT_BITS];
  const int bins = 1 << nbits;
  for (int i = threadIdx.x; i < bins; i += 1024) cnt[i] = 0;
  __syncthreads();
  const int64_t a1 = min(N, (blockIdx.x + 1) * chunk);
  for (int64_t a = blockIdx.x * chunk + threadIdx.x; a < a1; a += 1024) {
    const uint32_t k = FIRST ? row_of(ids[a], begin, rows) : key[a];
    atomicAdd(&cnt[(k >> shift) & (bins - 1)], 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += 1024) count[blockIdx.x * bins + i] = cnt[i];
}

// And this one places them: a digit's first place in the block is the tokens of
// lower digits and those of earlier blocks; within the block, waves by their
// order and lanes by theirs.
template <bool FIRST>
__global__ __launch_bounds__(64 * SORT_W) void embed_place_kernel(
    const int32_t* __restrict__ ids, const uint32_t* __restrict__ key_in,
    const int32_t* __restrict__ tok_in, int64_t N, int64_t chunk, int64_t begin, int64_t rows,
    int shift, int nbits, const int32_t* __restrict__ count, uint32_t* __restrict__ key,
    int32_t* __restrict__ tok) {
  __shared__ int cnt[SORT_W << SORT_BITS];
  __shared__ int wsum[SORT_W];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, bins = 1 << nbits;
  const int blocks = gridDim.x;
  for (int i = tid; i < SORT_W * bins; i += 64 * SORT_W) cnt[i] = 0;
  int total = 0, before = 0;
  if (tid < bins) {
#pragma unroll 16
    for (int b = 0; b < blocks; ++b) {
      const int c = count[b * bins + tid];
      total += c;
      before += b < static_cast<int>(blockIdx.x) ? c : 0;
    }
  }
  __syncthreads();
  int* mine = cnt + w * bins;
  const int64_t slice = chunk / SORT_W;  // a multiple of 64
  const int64_t base = blockIdx.x * chunk + w * slice;
  const int64_t end = min(N, base + slice);
  for (int64_t a = base + lane; a < end; a += 64) {
    const uint32_t k = FIRST ? row_of(ids[a], begin, rows) : key_in[a];
    atomicAdd(&mine[(k >> shift) & (bins - 1)], 1);
  }
  const int first = scan_bins(total, wsum) + before;  // its barrier: the counts are whole
  if (tid < bins) {
    int run = first;
    for (int u = 0; u < SORT_W; ++u) {
      const int c = cnt[u * bins + tid];
      cnt[u * bins + tid] = run;
      run += c;
    }
  }
  __syncthreads();
  for (int64_t a0 = base; a0 < end; a0 += 64) {
    const int64_t a = a0 + lane;
    const bool in = a < end;
    uint32_t k = 0;
    if (in) k = FIRST ? row_of(ids[a], begin, rows) : key_in[a];
    const uint32_t dg = (k >> shift) & (bins - 1);
    const uint64_t same = same_digit(dg, nbits, in);
    if (in) {
      const int at = mine[dg];
      const int p = at + lower_lanes(same, lane);
      key[p] = k;
      tok[p] = FIRST ? static_cast<int32_t>(a) : tok_in[a];
      if ((same >> lane) == 1ull) mine[dg] = at + __popcll(same);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// ---------------------------------------------------------------- gradient
// A team of 2^s lanes sums the rows of dy of one piece's tokens over 8 * 2^s
// columns (a slab).  part [pieces][2][H]: sums of the run that comes from the
// piece before (0) and of the run that goes on into the next (1).
// Workgroups from `sums` on write the zeros of rows without tokens.
__global__ __launch_bounds__(256) void embed_sum_kernel(
    const uint32_t* __restrict__ key, const int32_t* __restrict__ tok,
    const uint16_t* __restrict__ dy, int64_t N, int H, int64_t rows, float scale, int s, int slabs,
    int piece, int64_t sums, float* __restrict__ part, uint16_t* __restrict__ dw) {
  const int nch = H >> 3, lanes = 1 << s, l = threadIdx.x & (lanes - 1);
  const int team = threadIdx.x >> s, teams = 256 >> s;
  if (blockIdx.x >= sums) {
    __shared__ int there[ZERO_ROWS];
    const int64_t row0 = (blockIdx.x - sums) * ZERO_ROWS;
    if (threadIdx.x < ZERO_ROWS) {
      const int64_t r = row0 + threadIdx.x;
      int64_t lo = 0, n = N;  // the first place with a key of r or more
      while (n > 0) {
        const int64_t half = n >> 1;
        if (key[lo + half] < r) {
          lo += half + 1;
          n -= half + 1;
        } else {
          n = half;
        }
      }
      there[threadIdx.x] = r >= rows || (lo < N && key[lo] == r);
    }
    __syncthreads();
    for (int i = team; i < ZERO_ROWS; i += teams) {
      if (there[i]) continue;
      uint4* out = reinterpret_cast<uint4*>(dw + (row0 + i) * H);
      for (int c = l; c < nch; c += lanes) out[c] = make_uint4(0, 0, 0, 0);
    }
    return;
  }
  const int64_t id = static_cast<int64_t>(blockIdx.x) * teams + team;
  const int64_t pc = id / slabs;
  const int c = static_cast<int>(id - pc * slabs) * lanes + l;
  const int64_t p0 = pc * piece, p1 = min(N, p0 + piece);
  if (p0 >= N || c >= nch) return;
  uint32_t cur = key[p0];
  if (cur >= rows) return;
  bool head = p0 > 0 && key[p0 - 1] == cur;
  float acc[8] = {};
  auto flush = [&](bool tail) {
    if (cur >= rows) return;
    if (!head && !tail) {
      float f[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) f[q] = acc[q] * scale;
      reinterpret_cast<uint4*>(dw + static_cast<int64_t>(cur) * H)[c] = pack8(f);
    } else {
      float4* o = reinterpret_cast<float4*>(part + (pc * 2 + (head ? 0 : 1)) * H + 8 * c);
      o[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
      o[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
    }
  };
  constexpr int U = 8;
  for (int64_t p = p0; p < p1; p += U) {
    uint32_t k[U];
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      k[u] = p + u < p1 ? key[p + u] : static_cast<uint32_t>(rows);
      if (k[u] < rows)
        v[u] = reinterpret_cast<const uint4*>(dy + static_cast<int64_t>(tok[p + u]) * H)[c];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p + u < p1) {
        if (k[u] != cur) {
          flush(false);
          cur = k[u];
          head = false;
#pragma unroll
          for (int q = 0; q < 8; ++q) acc[q] = 0.0f;
        }
        if (k[u] < rows) {
          float f[8];
          unpack8(v[u], f);
#pragma unroll
          for (int q = 0; q < 8; ++q) acc[q] += f[q];
        }
      }
    }
  }
  flush(p1 < N && key[p1] == cur);
}

// The runs that pass the end of the piece they begin in: one workgroup a piece
// and slab; its teams take every teams-th of the run's pieces.
__global__ __launch_bounds__(256) void embed_join_kernel(
    const uint32_t* __restrict__ key, int64_t N, int H, int64_t rows, float scale, int s, int slabs,
    int piece, const float* __restrict__ part, uint16_t* __restrict__ dw) {
  __shared__ float sums[256 * 8];
  const int nch = H >> 3, lanes = 1 << s, l = threadIdx.x & (lanes - 1);
  const int team = threadIdx.x >> s, teams = 256 >> s;
  const int64_t pc = blockIdx.x / slabs;
  const int c = static_cast<int>(blockIdx.x - pc * slabs) * lanes + l;
  const int64_t p0 = pc * piece, p1 = p0 + piece;
  if (p1 >= N) return;
  const uint32_t k = key[p1];
  if (k >= rows || key[p1 - 1] != k) return;
  if (key[p0] == k && p0 > 0 && key[p0 - 1] == k) return;  // it began before
  int64_t more = 0;  // pieces after this one that begin in the run
  for (;;) {
    const int64_t at = (pc + 1 + more + (threadIdx.x & 63)) * piece;
    const uint64_t m = __ballot(at < N && key[at < N ? at : 0] == k);
    more += __popcll(m);
    if (m != ~0ull) break;
  }
  float acc[8] = {};
  if (c < nch) {
    for (int64_t i = team; i <= more; i += teams) {
      const float4* o = reinterpret_cast<const float4*>(
          part + ((pc + i) * 2 + (i == 0 ? 1 : 0)) * H + 8 * c);
      const float4 a = o[0], b = o[1];
      acc[0] += a.x; acc[1] += a.y; acc[2] += a.z; acc[3] += a.w;
      acc[4] += b.x; acc[5] += b.y; acc[6] += b.z; acc[7] += b.w;
    }
  }
#pragma unroll
  for (int q = 0; q < 8; ++q) sums[threadIdx.x * 8 + q] = acc[q];
  __syncthreads();
  if (team == 0 && c < nch) {
    for (int u = 1; u < teams; ++u)
#pragma unroll
      for (int q = 0; q < 8; ++q) acc[q] += sums[(u * lanes + l) * 8 + q];
    float f[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) f[q] = acc[q] * scale;
    reinterpret_cast<uint4*>(dw + static_cast<int64_t>(k) * H)[c] = pack8(f);
  }
}

__global__ __launch_bounds__(256) void embed_zero_kernel(int64_t n, uint4* __restrict__ dw) {
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n;
       i += static_cast<int64_t>(gridDim.x) * 256)
    dw[i] = make_uint4(0, 0, 0, 0);
}

// Lanes of a team, as a power of two: a row's chunks, within a wave.
int team_shift(int H) {
  int s = 0;
  while (s < 6 && (8 << s) < H) ++s;
  return s;
}

struct Plan {
  int s, slabs, piece, nbits, passes;
  int64_t pieces, blocks, chunk;
  size_t key[2], tok[2], count, part, bytes;
};

Plan plan_bwd(int64_t N, int H, int64_t rows) {
  Plan p{};
  p.s = team_shift(H);
  p.slabs = static_cast<int>(ceil_div(H, 8 << p.s));
  // tokens of a piece: enough teams to fill the chip first
  p.piece = 8;
  while (p.piece < 64 && ceil_div(N, 2 * p.piece) * p.slabs << p.s >= 8192 * 64) p.piece *= 2;
  p.pieces = ceil_div(N, p.piece);
  int bits = 1;
  while ((rows >> bits) > 0) ++bits;  // keys 0 .. rows
  p.passes = static_cast<int>(ceil_div(bits, SORT_BITS));
  p.nbits = static_cast<int>(ceil_div(bits, p.passes));
  const int64_t most = N <= (int64_t{1} << 20) ? SORT_BLOCKS : 4 * SORT_BLOCKS;
  p.blocks = std::clamp<int64_t>(ceil_div(N, 64 * SORT_W), 1, most);
  p.chunk = std::max<int64_t>(1, ceil_div(ceil_div(N, p.blocks), 64 * SORT_W)) * (64 * SORT_W);
  p.blocks = std::max<int64_t>(1, ceil_div(N, p.chunk));
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align_up(bytes, 256);
    return here;
  };
  const bool small = N <= SORT_SMALL;
  for (int i = 0; i < (small ? 1 : 2); ++i) {
    p.key[i] = take(4 * static_cast<size_t>(N));
    p.tok[i] = take(4 * static_cast<size_t>(N));
  }
  if (!small) p.count = take(4 * static_cast<size_t>(p.blocks) << p.nbits);
  p.part = take(8 * static_cast<size_t>(p.pieces) * H);
  p.bytes = at;
  return p;
}

}  // namespace

hipError_t launch_embed_fwd(const int32_t* ids, const uint16_t* w, int64_t N, int H, int64_t begin,
                            int64_t rows, float scale, uint16_t* y, hipStream_t s) {
  if (N == 0) return hipSuccess;
  const int sh = team_shift(H);
  const unsigned grid = static_cast<unsigned>(std::min<int64_t>(ceil_div(N << sh, 256), 1 << 20));
  prof_begin(K_EMBED, s);
  embed_fwd_kernel<<<grid, 256, 0, s>>>(ids, w, N, H, begin, rows, scale, sh, y);
  prof_end(K_EMBED, s);
  return hipGetLastError();
}

size_t embed_bwd_ws_bytes(int64_t N, int H, int64_t rows) { return plan_bwd(N, H, rows).bytes; }

hipError_t launch_embed_bwd(const int32_t* ids, const uint16_t* dy, int64_t N, int H, int64_t begin,
                            int64_t rows, float scale, uint16_t* dw, void* ws, hipStream_t s) {
  if (N == 0) {
    const int64_t n = rows * H / 8;
    prof_begin(K_EMBED_SUM, s);
    embed_zero_kernel<<<static_cast<unsigned>(std::min<int64_t>(ceil_div(n, 256), 1 << 20)), 256, 0,
                        s>>>(n, reinterpret_cast<uint4*>(dw));
    prof_end(K_EMBED_SUM, s);
    return hipGetLastError();
  }
  const Plan p = plan_bwd(N, H, rows);
  char* at = static_cast<char*>(ws);
  auto key = [&](int i) { return reinterpret_cast<uint32_t*>(at + p.key[i]); };
  auto tok = [&](int i) { return reinterpret_cast<int32_t*>(at + p.tok[i]); };
  int last = 0;
  prof_begin(K_EMBED_SORT, s);
  if (N <= SORT_SMALL) {
    embed_sort_small_kernel<<<1, 64 * SORT_W, 0, s>>>(ids, static_cast<int>(N), begin, rows,
                                                      p.passes, p.nbits, key(0), tok(0));
  } else {
    int32_t* count = reinterpret_cast<int32_t*>(at + p.count);
    const unsigned grid = static_cast<unsigned>(p.blocks);
    embed_count_kernel<true><<<grid, 1024, 0, s>>>(ids, nullptr, N, p.chunk, begin, rows, 0,
                                                   p.nbits, count);
    embed_place_kernel<true><<<grid, 64 * SORT_W, 0, s>>>(ids, nullptr, nullptr, N, p.chunk, begin,
                                                          rows, 0, p.nbits, count, key(0), tok(0));
    for (int i = 1; i < p.passes; ++i, last ^= 1) {
      embed_count_kernel<false><<<grid, 1024, 0, s>>>(nullptr, key(last), N, p.chunk, begin, rows,
                                                      i * p.nbits, p.nbits, count);
      embed_place_kernel<false><<<grid, 64 * SORT_W, 0, s>>>(
          nullptr, key(last), tok(last), N, p.chunk, begin, rows, i * p.nbits, p.nbits, count,
          key(last ^ 1), tok(last ^ 1));
    }
  }
  prof_end(K_EMBED_SORT, s);
  float* part = reinterpret_cast<float*>(at + p.part);
  const int64_t sums = ceil_div(p.pieces * p.slabs << p.s, 256);
  prof_begin(K_EMBED_SUM, s);
  embed_sum_kernel<<<static_cast<unsigned>(sums + ceil_div(rows, ZERO_ROWS)), 256, 0, s>>>(
      key(last), tok(last), dy, N, H, rows, scale, p.s, p.slabs, p.piece, sums, part, dw);
  embed_join_kernel<<<static_cast<unsigned>(p.pieces * p.slabs), 256, 0, s>>>(
      key(last), N, H, rows, scale, p.s, p.slabs, p.piece, part, dw);
  prof_end(K_EMBED_SUM, s);
  return hipGetLastError();
}

}  // namespace moe
