// Embedding of tokens and its weight gradient (gfx950).
//   y[t] = bf16(scale W[ids[t] - begin]),   0 where that is no row of this rank;
//   dW[v] = bf16(scale sum of dy[t] over t with ids[t] - begin = v), t ascending.
// The gradient sorts the tokens by row (stable, so that sums have one order), then
// cuts the sorted list into pieces of equal length, so that a frequent word costs
// no wave more than a rare one: a run of one row inside a piece is summed in
// registers and written; one that passes a piece's end leaves fp32 partial sums,
// which are joined in a fixed order (each team of lanes takes every so many-th, then the
// teams are added up).  Rows without tokens are written as zeros by workgroups that look
// them up in the sorted list.  Both directions are bound by the HBM stream of their rows,
// the gradient mostly by writing dW.  65536 tokens by Zipf's law, H = 4096, 200,000 rows:
// the forward 130 us (5.5 TB/s), sorting 25, sums and zeros 375 (5.8 TB/s), joining 18;
// the forward takes 175 right after such a gradient and the gradient 30 less than
// otherwise (its 1.6 GB are still on their way to memory when the next kernel starts);
// 2000 rows: sums and joining 121.  With few tokens it is the launches and their
// latency (256 tokens, H = 128: 3 us, then 5, 4 and 3).
#include <algorithm>

#include "common.h"

namespace moe {
namespace {

constexpr int SORT_W = 16;        // waves of a sorting workgroup
constexpr int SORT_SMALL = 8192;  // tokens that one workgroup sorts
constexpr int SORT_BITS = 10;     // widest digit: two of them sort up to 2^20 - 1 rows
constexpr int SORT_BLOCKS = 64;   // workgroups of a sorting pass, up to 2^20 tokens
constexpr int ZERO_ROWS = 32;     // rows looked up by a workgroup

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
        if (c0 + u * lanes < nch)
          store_stream(dst + c0 + u * lanes, there ? pack8(f) : make_uint4(0, 0, 0, 0));
      }
    }
  }
}

// ------------------------------------------------------------------ sorting
// The lanes of a wave that have this lane's digit (nbits of it).  Four vector
// instructions a bit: they bound the sort of one workgroup.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, int nbits, bool in) {
  const uint64_t all = __ballot(in);
  uint32_t lo = static_cast<uint32_t>(all), hi = static_cast<uint32_t>(all >> 32);
  for (int b = 0; b < nbits; ++b) {
    const uint32_t mine = static_cast<uint32_t>(__builtin_amdgcn_sbfe(static_cast<int>(digit), b, 1));
    const uint64_t bal = __ballot(mine != 0);
    lo &= ~(static_cast<uint32_t>(bal) ^ mine);
    hi &= ~(static_cast<uint32_t>(bal >> 32) ^ mine);
  }
  return static_cast<uint64_t>(hi) << 32 | lo;
}
__device__ __forceinline__ int lower_lanes(uint64_t m, int lane) {
  return __popcll(m & (lane == 0 ? 0ull : (~0ull >> (64 - lane))));
}

// Exclusive sums over at most 1024 values, one a thread of the workgroup's first (v = 0
// beyond): every thread calls it.
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

// A digit's counts of the workgroup's waves, all read before any is overwritten (one
// by one, each load would wait for the store before it), and their sum; then the
// waves' first places, from `first` on.
__device__ __forceinline__ int wave_counts(int (&c)[SORT_W], const int* cnt, int bins) {
  int sum = 0;
#pragma unroll
  for (int u = 0; u < SORT_W; ++u) c[u] = cnt[u * bins];
#pragma unroll
  for (int u = 0; u < SORT_W; ++u) sum += c[u];
  return sum;
}
__device__ __forceinline__ void wave_places(const int (&c)[SORT_W], int* cnt, int bins, int first) {
#pragma unroll
  for (int u = 0; u < SORT_W; ++u) {
    cnt[u * bins] = first;
    first += c[u];
  }
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
    int c[SORT_W], run = 0;
    if (tid < bins) run = wave_counts(c, cnt + tid, bins);
    const int first = scan_bins(run, wsum);
    if (tid < bins) wave_places(c, cnt + tid, bins, first);
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
    int c[SORT_W];
    wave_counts(c, cnt + tid, bins);
    wave_places(c, cnt + tid, bins, first);
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
// The first place with a key of r or more: a whole wave looks, 64 places a step.
__device__ __forceinline__ int64_t first_not_below(const uint32_t* __restrict__ key, int64_t n,
                                                   int64_t r) {
  const int lane = lane_id();
  int64_t lo = 0;
  while (n > 0) {
    const int64_t step = (n + 63) >> 6;
    const int64_t probe = lo + min((lane + 1) * step, n) - 1;
    const int below = __popcll(__ballot(key[probe] < r));
    if (below == 64) return lo + n;
    lo += below * step;
    n = min(step, n - below * step) - 1;  // the probe itself is not below
  }
  return lo;
}

// A team of 2^s lanes sums the rows of dy of one piece's tokens over 8 * 2^s
// columns (a slab).  part [pieces][2][H]: sums of the run that comes from the
// piece before (0) and of the run that goes on into the next (1).
// Workgroups from `sums` on write the zeros of rows without tokens.
// WAVE: a team is a wave (s = 6), and keys and tokens are scalars of it.
template <bool WAVE>
__global__ __launch_bounds__(256) void embed_sum_kernel(
    const uint32_t* __restrict__ key, const int32_t* __restrict__ tok,
    const uint16_t* __restrict__ dy, int64_t N, int H, int64_t rows, float scale, int s, int slabs,
    int piece, int64_t sums, float* __restrict__ part, uint16_t* __restrict__ dw) {
  const int nch = H >> 3, lanes = WAVE ? 64 : 1 << s, l = threadIdx.x & (lanes - 1);
  const int team = WAVE ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : threadIdx.x >> s;
  const int teams = WAVE ? 4 : 256 >> s;
  if (blockIdx.x >= sums) {
    __shared__ int64_t ends[2];
    __shared__ int there[ZERO_ROWS];
    const int64_t row0 = (blockIdx.x - sums) * ZERO_ROWS;
    // the tokens of these rows lie between two places; each row looks between them
    if (threadIdx.x < 128) {
      const int64_t at = first_not_below(key, N, row0 + (threadIdx.x < 64 ? 0 : ZERO_ROWS));
      if ((threadIdx.x & 63) == 0) ends[threadIdx.x >> 6] = at;
    }
    __syncthreads();
    if (threadIdx.x < ZERO_ROWS) {
      const int64_t r = row0 + threadIdx.x;
      int64_t lo = ends[0], n = ends[1] - lo;
      while (n > 0) {
        const int64_t half = n >> 1;
        if (key[lo + half] < r) {
          lo += half + 1;
          n -= half + 1;
        } else {
          n = half;
        }
      }
      there[threadIdx.x] = r >= rows || (lo < ends[1] && key[lo] == r);
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
  const int64_t p0 = pc * piece;
  if (p0 >= N || (!WAVE && c >= nch)) return;
  const int n = static_cast<int>(min<int64_t>(N - p0, piece));
  // what lies beyond the row's end is read from its first column, and not written
  const uint4* col = reinterpret_cast<const uint4*>(dy) + (c < nch ? c : 0);
  uint32_t kl = 0;
  int tl = 0;
  if constexpr (WAVE) {  // a lane a token (pieces are 64 at most)
    kl = key[p0 + min(l, n - 1)];
    tl = tok[p0 + min(l, n - 1)];
  }
  auto key_at = [&](int i) -> uint32_t {
    if constexpr (WAVE) return __builtin_amdgcn_readlane(kl, i);
    else return key[p0 + min(i, n - 1)];
  };
  auto tok_at = [&](int i) -> int {
    if constexpr (WAVE) return __builtin_amdgcn_readlane(tl, i);
    else return tok[p0 + min(i, n - 1)];
  };
  uint32_t cur = key_at(0);
  if (cur >= rows) return;
  bool head = p0 > 0 && key[p0 - 1] == cur;
  float acc[8] = {};
  auto flush = [&](bool tail) {
    if (cur >= rows || (WAVE && c >= nch)) return;
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
  // U rows on their way while U are summed (keys and rows asked for one by one, with
  // a test before each, made 104 us 170); those past the list's end repeat its last
  // one without being summed.  U = 8 is no faster on whole waves, and on narrow rows,
  // where it takes 130 registers, slower (20 us: 37)
  constexpr int U = 4;
  uint32_t k[2][U];
  uint4 v[2][U];
  auto fetch = [&](int i, int b) {
    int t[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      k[b][u] = key_at(i + u);
      t[u] = tok_at(i + u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      v[b][u] = load_stream(col + static_cast<int64_t>(t[u]) * nch);
  };
  auto add = [&](int i, int b) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u < n) {
        if (k[b][u] != cur) {
          flush(false);
          cur = k[b][u];
          head = false;
#pragma unroll
          for (int q = 0; q < 8; ++q) acc[q] = 0.0f;
        }
        float f[8];
        unpack8(v[b][u], f);
#pragma unroll
        for (int q = 0; q < 8; ++q) acc[q] += f[q];
      }
    }
  };
  fetch(0, 0);
  for (int i = 0; i < n; i += 2 * U) {
    if (i + U < n) fetch(i + U, 1);
    add(i, 0);
    if (i + 2 * U < n) fetch(i + 2 * U, 0);
    if (i + U < n) add(i + U, 1);
  }
  flush(p0 + n < N && key[p0 + n] == cur);
}

// The runs that pass the end of the piece they begin in: one workgroup a piece and
// slab; its teams take every teams-th of the run's pieces, eight loads at a time.
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
  // all at once, for the many that end here
  const int64_t at0 = (pc + 1 + (threadIdx.x & 63)) * piece;
  const uint32_t k = key[p1], end = key[p1 - 1], first = key[p0], earlier = key[p0 > 0 ? p0 - 1 : 0];
  const uint32_t probe = key[at0 < N ? at0 : 0];
  if (k >= rows || end != k) return;
  if (first == k && p0 > 0 && earlier == k) return;  // it began before
  // pieces after this one that begin in the run
  uint64_t m = __ballot(at0 < N && probe == k);
  int64_t more = __popcll(m);
  while (m == ~0ull) {
    const int64_t at = at0 + more * piece;
    m = __ballot(at < N && key[at < N ? at : 0] == k);
    more += __popcll(m);
  }
  float acc[8] = {};
  if (c < nch) {
    constexpr int B = 8;
    for (int64_t i0 = team; i0 <= more; i0 += B * teams) {
      float4 a[B], b[B];
#pragma unroll
      for (int u = 0; u < B; ++u) {
        const int64_t i = i0 + u * teams;
        a[u] = b[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (i <= more) {
          const float4* o = reinterpret_cast<const float4*>(
              part + ((pc + i) * 2 + (i == 0 ? 1 : 0)) * H + 8 * c);
          a[u] = o[0];
          b[u] = o[1];
        }
      }
#pragma unroll
      for (int u = 0; u < B; ++u) {
        acc[0] += a[u].x; acc[1] += a[u].y; acc[2] += a[u].z; acc[3] += a[u].w;
        acc[4] += b[u].x; acc[5] += b[u].y; acc[6] += b[u].z; acc[7] += b[u].w;
      }
    }
  }
#pragma unroll
  for (int q = 0; q < 8; ++q) sums[threadIdx.x * 8 + q] = acc[q];
  __syncthreads();
  if (team == 0 && c < nch) {
    const int some = static_cast<int>(min<int64_t>(teams, more + 1));
    for (int u = 1; u < some; ++u)
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
  // tokens of a piece: some 1024 waves come first, longer pieces then (they leave fewer
  // runs to join: 16384 tokens, half of them one word, H = 2048, over 1000 rows take
  // 38 us, with 8192 waves of 8 tokens 68; with 256 waves 4096 tokens take 36 for 30)
  p.piece = 8;
  while (p.piece < 64 && ceil_div(N, 2 * p.piece) * p.slabs << p.s >= 1024 * 64) p.piece *= 2;
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
  const unsigned grid = static_cast<unsigned>(sums + ceil_div(rows, ZERO_ROWS));
  if (p.s == 6)
    embed_sum_kernel<true><<<grid, 256, 0, s>>>(key(last), tok(last), dy, N, H, rows, scale, p.s,
                                                p.slabs, p.piece, sums, part, dw);
  else
    embed_sum_kernel<false><<<grid, 256, 0, s>>>(key(last), tok(last), dy, N, H, rows, scale, p.s,
                                                 p.slabs, p.piece, sums, part, dw);
  if (p.pieces > 1)
    embed_join_kernel<<<static_cast<unsigned>((p.pieces - 1) * p.slabs), 256, 0, s>>>(
        key(last), N, H, rows, scale, p.s, p.slabs, p.piece, part, dw);
  prof_end(K_EMBED_SUM, s);
  return hipGetLastError();
}

}  // namespace moe
