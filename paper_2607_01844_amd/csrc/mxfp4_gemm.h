// Grouped expert products on MXFP4 operands (gfx950's scaled matrix
// instruction): 4-bit values (e2m1) in blocks of 32 along the contraction, one
// power-of-two scale byte a block.
//
// The tile kernel is the shape of the bf16 one's K-contiguous operands
// (gemm_kernel.h): a 256 x 256 tile on eight waves (128 rows x 64 columns
// each; or 128 x 128 on four, two workgroups a CU), operands straight to LDS,
// fragments read between the matrix instructions.  One v_mfma_scale_f32_32x32x64
// takes 16 bytes a lane and operand, as the bf16 instruction does, and as many
// cycles, for four times the products: a step of 128 bytes a row is 256 k.
// Beside the values a step has 8 scale bytes a row, a contiguous 2 KiB of the
// layout that the quantiser writes: [256 k][row][8], the four even blocks' bytes
// first, so that lane l (row l % 32, blocks of half l / 32) takes its four
// sub-steps' scales as one dword and each instruction picks its byte.
//   Both operands have two slots each (128 KiB, and 8 KiB of scales; a third for
// the weights, as the bf16 kernel has, does not fit beside the scales).  B's
// fragments of a whole step are read in its first sub-step, so that a barrier frees
// B's slot there and B is loaded a step and a half ahead of its use; A's slot is
// free before the last sub-step, whose products run from registers while the
// next step's first fragments are read.  The loads run on their own walk over
// the tiles, so tiles follow one another without a pause in the stream, however
// short they are.
//   Measured, 128 experts of 512 rows, d = 4096, f = 1536, gate/up: 473 us (565 in
// a sustained run, when the card lowers its clock) for 1.65e12 operations, 3.5e15 a
// second.  Parts of the same loop with the rest taken out: the products from
// registers 226 us more than the 74 that epilogues and tile changes take (48 % of
// the cycles of the whole kernel; on zeros, at a higher clock, the whole takes
// 403), the loads 250 more, the fragment reads 90 more.  So it is neither the
// matrix cores, nor the loads, nor LDS alone, but all three in turn under one power
// limit: half a step more between A's loads and their use (its rows read half by
// half), or other orders of the steps over K, changed nothing.  With 16 rows an
// expert the kernel streams its weights: 196 MB in 29 us, 6.8 TB/s.
#pragma once

#include "gemm_kernel.h"

namespace moe {
namespace gemm {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4v __attribute__((ext_vector_type(4)));

enum MxMode { MX_GATE_UP = 0, MX_DOWN = 1 };

// An MXFP4 matrix of `rows` rows along K: values [rows][kq] (kq = 16 bytes a
// block), scales [ceil(K / 256)][rows][8].
struct MxMat {
  const uint8_t* q;
  const uint8_t* s;
};

struct MxArgs {
  MxMat a;                // activations: x (of x_rows rows) or act (of cap rows)
  MxMat b0, b1;           // weights of expert 0: gate and up, or down
  const int32_t* a_tok;   // row of a.q for each permuted row (null: the row itself)
  int64_t a_rows;         // rows of a.s
  int64_t a_bytes;        // of a.q
  uint8_t* act_q;         // gate/up: silu(gate) up in MXFP4, cap rows along f
  uint8_t* act_s;
  int64_t cap;
  uint16_t* y;            // down: [cap][d] bf16
  GemmArgs t;             // the tile walk's: offsets, tables, E_loc, d, f, NT
};

template <int S>
struct MxGeom {
  static constexpr int UNIT = S * 128;  // one operand, one step
  static constexpr int SUNIT = S * 8;   // its scales
  static constexpr int NWAVE = S / 32, NTHR = 64 * NWAVE, AIM = S / 64;
  static constexpr int PATCH = 2048;    // per wave, of the bf16 output
  static constexpr int SCALES = 4 * UNIT, PATCHES = SCALES + 4 * SUNIT;
  static constexpr int TOKENS = PATCHES + NWAVE * PATCH;  // tokens of each wave's rows
  static constexpr int LDS = TOKENS + NWAVE * 256;        // 154 KiB, or 77 KiB
};

// 4 bytes per lane, global -> LDS (see load_lds16)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds4(const i32x4& rsrc, uint32_t voff, uint32_t lds) {
  i32x4 r;
  r[0] = __builtin_amdgcn_readfirstlane(rsrc[0]);
  r[1] = __builtin_amdgcn_readfirstlane(rsrc[1]);
  r[2] = __builtin_amdgcn_readfirstlane(rsrc[2]);
  r[3] = __builtin_amdgcn_readfirstlane(rsrc[3]);
  const uint32_t l = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds"
               :
               : "s"(l), "v"(voff), "s"(r)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// This wave's 32 rows of one operand of a tile, values and scales: load q of
// step j fills tile rows 32 w + 8 q .. + 7 (16-byte chunk c of row r at
// (c ^ ((r / 2) % 8)), as KOperand's), one dword a lane the rows' scale bytes.
struct MxStream {
  i32x4 rs;
  uint32_t voff[4];
  uint64_t sbase;   // scales of the wave's first row at step 0
  uint32_t srange;  // bytes of scales from there to the last row's
  uint64_t sstep;   // bytes from one step's scales to the next's
  int chunks;       // valid 16-byte chunks of a row
  // row r (0 .. 31) of the wave is valid below `rows` and at off(r) * kq from p
  template <typename F>
  __device__ __forceinline__ void setup(const uint8_t* p, int64_t bytes, int kq, int rows, F&& off,
                                        const uint8_t* s, int64_t s_rows, int64_t s_row0, int lane) {
    rs = make_rsrc(p, bytes);
    chunks = kq / 16;
    const int rl = lane >> 3;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int row = 8 * q + rl;
      const int lc = (lane & 7) ^ ((row >> 1) & 7);
      voff[q] = row < rows ? static_cast<uint32_t>(off(row)) * static_cast<uint32_t>(kq) +
                                 static_cast<uint32_t>(16 * lc)
                           : OOB;
    }
    sbase = reinterpret_cast<uint64_t>(s) + static_cast<uint64_t>(s_row0) * 8;
    sstep = static_cast<uint64_t>(s_rows) * 8;
    const int64_t left = s_rows - s_row0;
    srange = left <= 0 || rows <= 0 ? 0u : static_cast<uint32_t>(left < 32 ? left : 32) * 8u;
  }
  // nothing (every lane out of range: zeros), after the last tile
  __device__ __forceinline__ void none() {
    chunks = 0;
    srange = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) voff[q] = OOB;
  }
  // Step j's values into the LDS unit at `u`.  TAIL: chunks past the row's end
  // read as zeros; of two operands one that does is enough, since the other's
  // then meet zeros (codes are finite whatever the bytes).  No branches: one in
  // the middle of a step would let the compiler gather the step's matrix
  // instructions behind it.
  template <bool TAIL>
  __device__ __forceinline__ void values(int j, uint32_t u, int w, int lane) const {
    const uint32_t kb = static_cast<uint32_t>(j) * 128u;
    if constexpr (TAIL) {
      const int lc0 = (lane & 7) ^ (lane >> 4);  // chunk of loads 0 and 2; of 1 and 3 lc0 ^ 4
      const bool in[2] = {lc0 < chunks - 8 * j, (lc0 ^ 4) < chunks - 8 * j};
#pragma unroll
      for (int q = 0; q < 4; ++q) load_lds16(rs, in[q & 1] ? voff[q] + kb : OOB, u + (4 * w + q) * 1024);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) load_lds16(rs, voff[q] + kb, u + (4 * w + q) * 1024);
    }
  }
  __device__ __forceinline__ void scales(int j, uint32_t u, int w, int lane) const {
    const uint64_t a = sbase + static_cast<uint64_t>(j) * sstep;
    i32x4 r;
    r[0] = static_cast<int>(a & 0xffffffffu);
    r[1] = static_cast<int>((a >> 32) & 0xffffu);
    r[2] = static_cast<int>(srange);
    r[3] = 0x00020000;
    load_lds4(r, static_cast<uint32_t>(4 * lane), u + w * 256);
  }
};

// Lanes below 32 get the pair (a of their own, a of lane + 32), the others (b of
// lane - 32, b of their own).
__device__ __forceinline__ uint2 swap_halves(uint32_t a, uint32_t b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  return make_uint2(r[0], r[1]);
}
// Accumulators that have to be there at this point: keeps the matrix
// instructions before it from being moved behind the branches that follow.
__device__ __forceinline__ void pin(f32x16& v) { asm volatile("" : "+v"(v)); }

// One tile: rows [row0, row0 + rows) (permuted rows, at most 32 h) of expert e,
// output columns from n0.
struct MxTile {
  int valid, e, row0, rows, h, n0;
};

// The tiles of one workgroup, in the order of the bf16 row-grouped products'
// (TileIter), 64 at a time: lane i finds tile 64 b + i once, and a tile is read
// from the lanes when its turn comes.  (Found one by one, with a chain of
// scalar loads each, a tile took 4000 cycles of a gate/up product's 60,000.)
template <int S, bool DUAL>
struct MxList {
  int L0, stride, count;  // first tile, step, number of this workgroup's tiles
  int e, row0, rows, h, n0;  // of lane's tile
  __device__ __forceinline__ void init(int total) {
    const int xcd = blockIdx.x % NXCD;
    stride = gridDim.x / NXCD;
    const int per = (total + NXCD - 1) / NXCD;
    L0 = xcd * per + blockIdx.x / NXCD;
    const int end = min((xcd + 1) * per, total);
    count = L0 < end ? (end - 1 - L0) / stride + 1 : 0;
  }
  // tiles from, from + 1, ...; mt(i), off(i): entries of the tables
  template <typename MT, typename OFF>
  __device__ __forceinline__ void fill(int from, int E_loc, int NT, int lane, MT&& mt, OFF&& off) {
    const int i = min(from + lane, count - 1);
    const int L = L0 + i * stride;
    int lo = 0, hi = E_loc;
    while (hi - lo > 1) {  // the same number of turns in every lane, up to one
      const int mid = (lo + hi) >> 1;
      if (mt(mid) * NT <= L) lo = mid; else hi = mid;
    }
    const int m = mt(lo), mts = mt(lo + 1) - m;
    const int seg = off(lo), ne = off(lo + 1) - seg;
    int tm, tn;
    tile_pos<4>(L - m * NT, mts, NT, tm, tn);
    e = lo;
    h = tile_blocks(ne, mts);
    const int m0 = tm * 32 * h;
    row0 = seg + m0;
    rows = min(ne - m0, 32 * h);
    n0 = tn * (DUAL ? S / 2 : S);
  }
  __device__ __forceinline__ MxTile get(int i) const {
    auto at = [i](int v) { return __builtin_amdgcn_readlane(v, i & 63); };
    return MxTile{i < count, at(e), at(row0), at(rows), at(h), at(n0)};
  }
};

// 4-bit codes of a pair into byte SEL of `old`
template <int SEL>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t old, float a, float b, float scale) {
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, scale, SEL));
}
// Scale byte of a block whose largest magnitude has these fp32 bits: its
// exponent less that of 4 (the largest value's, 6 = 1.5 * 4), 255 for NaN and
// infinities.
__device__ __forceinline__ uint32_t mx_scale(uint32_t abs_bits) {
  const uint32_t e = abs_bits >> 23;
  return e == 255u ? 255u : (e < 2u ? 2u : e) - 2u;
}
// Where the scale byte of block b lies in the 8 bytes of its 256 k.
__device__ __forceinline__ int mx_pos(int b) { return (b & 1) * 4 + ((b & 7) >> 1); }

template <int MODE, int S>
__global__ __launch_bounds__(MxGeom<S>::NTHR, 2) void mxfp4_gemm_kernel(MxArgs g) {
  using G = MxGeom<S>;
  constexpr bool DUAL = MODE == MX_GATE_UP;
  constexpr int UNIT = G::UNIT, SUNIT = G::SUNIT, NWAVE = G::NWAVE, AIM = G::AIM;
  __shared__ __align__(1024) char lds[G::LDS];
  lds_char* const ring = (lds_char*)(lds);
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(ring));
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = (w ^ (w >> 2)) & 1, wn = w >> 1;  // both wave rows on every SIMD
  const int d = g.t.d, f = g.t.f;
  const int K = DUAL ? d : f, N = DUAL ? f : d;
  const int kq = (K + 31) / 32 * 16, nk = (K + 255) / 256;
  const int64_t wbytes = static_cast<int64_t>(N) * kq, sbytes = static_cast<int64_t>(nk) * N * 8;

  // ------------------------------------------------------------ loads
  // They run ahead of the products, two steps of K: at most two tiles (of one
  // step), which wait here for their turn.
  MxList<S, DUAL> list;
  {
    // the tables pass through the ring, which is not in use yet
    int* const mt = reinterpret_cast<int*>(lds);
    int* const off = mt + g.t.E_loc + 1;
    for (int i = threadIdx.x; i <= g.t.E_loc; i += G::NTHR) {
      mt[i] = g.t.mt_start[i];
      off[i] = g.t.offsets[i];
    }
    __syncthreads();
    list.init(__builtin_amdgcn_readfirstlane(mt[g.t.E_loc] * g.t.NT));
    if (list.count > 0)
      list.fill(0, g.t.E_loc, g.t.NT, lane, [&](int i) { return mt[i]; }, [&](int i) { return off[i]; });
    __syncthreads();
  }
  if (list.count == 0) return;
  MxTile q1{}, q2{};
  int queued = 0, li = 0;  // tiles waiting; the next one to load
  auto push = [&](const MxTile& t) __attribute__((always_inline)) {
    const bool one = queued == 0;
    auto pick = [one](int& a, int& b, int v) __attribute__((always_inline)) {
      a = one ? v : a;
      b = one ? b : v;
    };
    pick(q1.valid, q2.valid, t.valid);
    pick(q1.e, q2.e, t.e);
    pick(q1.row0, q2.row0, t.row0);
    pick(q1.rows, q2.rows, t.rows);
    pick(q1.h, q2.h, t.h);
    pick(q1.n0, q2.n0, t.n0);
    ++queued;
  };
  auto pop = [&]() __attribute__((always_inline)) {
    const MxTile t = q1;
    q1 = q2;
    --queued;
    return t;
  };
  // the tokens of this wave's rows of a tile, on their way to LDS
  auto load_tokens = [&](const MxTile& t, int lane) __attribute__((always_inline)) {
    const int rows = t.rows - 32 * w;
    load_lds4(make_rsrc(g.a_tok + t.row0 + 32 * w, 4 * min(rows, 32)), 4 * lane, lds0 + G::TOKENS + w * 256);
  };
  MxStream sa, sb;
  int lstep = 0;  // the next step to load of the loads' tile
  auto load_tile = [&]() __attribute__((always_inline)) {
    lstep = 0;
    if (li >= list.count) {
      sa.none();
      sb.none();
      if (queued < 2) push(MxTile{0, 0, 0, 0, 0, 0});  // the end (never more than one is read)
      return;
    }
    const int lane = opaque(threadIdx.x & 63);
    const bool fresh = (li & 63) == 0;
    if (fresh && li > 0)
      list.fill(li, g.t.E_loc, g.t.NT, lane, [&](int i) { return g.t.mt_start[i]; },
                [&](int i) { return g.t.offsets[i]; });
    const MxTile t = list.get(li);
    push(t);
    {
      const int rows = t.rows - 32 * w;
      const int64_t r0 = static_cast<int64_t>(t.row0) + 32 * w;
      if (g.a_tok != nullptr) {
        if (fresh) {
          load_tokens(t, lane);
          wait_vmcnt<0>();
        }
        const lds_char* tok = ring + G::TOKENS + w * 256;
        sa.setup(g.a.q, g.a_bytes, kq, rows,
                 [&](int r) { return *reinterpret_cast<const __attribute__((address_space(3))) int*>(tok + 4 * r); },
                 g.a.s, g.a_rows, r0, lane);
        ++li;
        // the next tile's, which the waits between land before its turn
        if (li < list.count && (li & 63) != 0) {
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          load_tokens(list.get(li), lane);
        }
      } else {
        sa.setup(g.a.q + r0 * kq, static_cast<int64_t>(rows) * kq, kq, rows, [](int r) { return r; }, g.a.s,
                 g.a_rows, r0, lane);
        ++li;
      }
    }
    {
      const bool up = DUAL && w >= NWAVE / 2;
      const int n0 = t.n0 + 32 * (DUAL ? w % (NWAVE / 2) : w);
      const MxMat& b = up ? g.b1 : g.b0;
      sb.setup(b.q + t.e * wbytes + static_cast<int64_t>(n0) * kq, static_cast<int64_t>(N - n0) * kq, kq, N - n0,
               [](int r) { return r; }, b.s + t.e * sbytes, N, n0, lane);
    }
  };
  // parts of the step `lstep` into slot `slot`
  auto load_a = [&](int slot) __attribute__((always_inline)) {
    sa.template values<false>(lstep, lds0 + slot * UNIT, w, 0);
  };
  auto load_b = [&](int slot) __attribute__((always_inline)) {
    sb.template values<true>(lstep, lds0 + (2 + slot) * UNIT, w, opaque(threadIdx.x & 63));
  };
  auto load_s = [&](int slot) __attribute__((always_inline)) {
    const int ln = opaque(threadIdx.x & 63);
    sa.scales(lstep, lds0 + G::SCALES + slot * SUNIT, w, ln);
    sb.scales(lstep, lds0 + G::SCALES + (2 + slot) * SUNIT, w, ln);
  };

  // --------------------------------------------------------- products
  int arow0 = 0, brow[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) brow[j] = DUAL ? j * (S / 2) + wn * 32 : wn * 64 + 32 * j;
  f32x16 acc[AIM][2];
  struct Scales {
    int a[AIM], b[2];
  };
  typedef const __attribute__((address_space(3))) i32x4v* lds_frag;
  i32x4v fa[2][AIM], fb[4][2];  // fragments: A's of a sub-step and the next, B's of a whole step
  int fl = lane;  // the lane, made opaque tile by tile: addresses of one row-block
                  // count are not kept live through another's loop
  auto load_fa = [&](int slot, auto SUB, auto I) __attribute__((always_inline)) {
    const lds_char* t = ring + slot * UNIT + (arow0 + 32 * I) * 128;
    fa[SUB & 1][I] = *reinterpret_cast<lds_frag>(t + koff(fl & 31, 2 * SUB + (fl >> 5)));
  };
  auto load_fb = [&](int slot, auto SUB, auto J) __attribute__((always_inline)) {
    const lds_char* t = ring + (2 + slot) * UNIT + brow[J] * 128;
    fb[SUB][J] = *reinterpret_cast<lds_frag>(t + koff(fl & 31, 2 * SUB + (fl >> 5)));
  };
  // the first sub-step's fragments of a step
  auto load_first = [&](int slot, auto AIC) __attribute__((always_inline)) {
    constexpr std::integral_constant<int, 0> Z{};
    load_fa(slot, Z, Z);
    load_fb(slot, Z, Z);
    load_fb(slot, Z, std::integral_constant<int, 1>{});
    static_for<AIM>([&](auto I) {
      if constexpr (I > 0 && I < AIC) load_fa(slot, Z, I);
    });
  };
  auto load_scales = [&](Scales& c, int slot, auto AIC) __attribute__((always_inline)) {
    const lds_char* s = ring + G::SCALES + slot * SUNIT + (fl & 31) * 8 + (fl >> 5) * 4;
    static_for<AIM>([&](auto I) {
      if constexpr (I < AIC)
        c.a[I] = *reinterpret_cast<const __attribute__((address_space(3))) int*>(s + (arow0 + 32 * I) * 8);
    });
#pragma unroll
    for (int j = 0; j < 2; ++j)
      c.b[j] = *reinterpret_cast<const __attribute__((address_space(3))) int*>(s + 2 * SUNIT + brow[j] * 8);
  };
  // FIRST: the tile's first sub-step, which starts from zero
  auto mma1 = [&](const Scales& c, auto SUB, auto T, auto FIRST) __attribute__((always_inline)) {
    constexpr int i = T / 2, j = T % 2, p = SUB & 1;
    const i32x8 bv = __builtin_shufflevector(fb[SUB][j], fb[SUB][j], 0, 1, 2, 3, -1, -1, -1, -1);
    const i32x8 av = __builtin_shufflevector(fa[p][i], fa[p][i], 0, 1, 2, 3, -1, -1, -1, -1);
    if constexpr (FIRST)
      acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(bv, av, f32x16{}, 4, 4, SUB, c.b[j], SUB, c.a[i]);
    else
      acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(bv, av, acc[i][j], 4, 4, SUB, c.b[j], SUB, c.a[i]);
    __builtin_amdgcn_sched_barrier(0);
  };
  // The 2 AI products of sub-step SUB.  Between them go the fragment reads of
  // A's next sub-step (and in sub-step 0 all the rest of B's), spread evenly,
  // and extra() halfway.
  auto mma_read = [&](const Scales& c, int slot, auto SUB, auto AIC, auto FIRST, auto&& extra) __attribute__((always_inline)) {
    constexpr int AI = AIC, n = AI + (SUB == 0 ? 6 : 0);  // reads
    static_for<2 * AI>([&](auto T) {
      mma1(c, SUB, T, FIRST);
      if constexpr (T == AI) {
        extra();
        __builtin_amdgcn_sched_barrier(0);
      }
      static_for<n>([&](auto R) {
        constexpr int r = R;
        if constexpr (r * 2 * AI / n == T) {
          // A's first fragment, B's (the next sub-step's first), then A's others
          if constexpr (SUB == 0) {
            if constexpr (r >= 1 && r < 7)
              load_fb(slot, std::integral_constant<int, 1 + (r - 1) / 2>{}, std::integral_constant<int, (r - 1) % 2>{});
            else load_fa(slot, std::integral_constant<int, 1>{}, std::integral_constant<int, r == 0 ? 0 : r - 6>{});
          } else {
            load_fa(slot, std::integral_constant<int, SUB + 1>{}, R);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      });
    });
  };

  // --------------------------------------------------------- epilogue
  // acc[i][j][4 q + u]: output row arow0 + 32 i + l32, column brow[j] + 8 q + 4 lh + u
  auto epilogue = [&](const MxTile& tl, int ai) __attribute__((always_inline)) {
    const int mvalid = tl.rows;
    const int64_t row0 = tl.row0;
    // lane-derived indices formed here, not kept live across the K loop
    const int lane = opaque(threadIdx.x & 63), l32 = lane & 31, lh = lane >> 5;
    static_for<AIM>([&](auto I) {
      constexpr int i = I;
      if (i >= ai) return;
      const int rb = arow0 + 32 * i;
      if constexpr (DUAL) {
        // The wave's 32 columns of a row are one block of the down product's
        // contraction: lanes l and l + 32 hold 16 each.
        const int col = tl.n0 + wn * 32;
        float a[16];
        uint32_t top = 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          // silu by the hardware's exponential and reciprocal (each within 2^-22)
          const float z = acc[i][0][r];
          a[r] = z * __builtin_amdgcn_rcpf(1.0f + __expf(-z)) * acc[i][1][r];
          top = max(top, __float_as_uint(a[r]) & 0x7fffffffu);
        }
        {
          const uint2 t = swap_halves(top, top);
          top = max(t.x, t.y);
        }
        const uint32_t e8 = mx_scale(top);
        const float sc = __uint_as_float(e8 << 23);
        uint32_t p[2];  // 16 bits of each of two q
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t v = 0;
          v = fp4_pair<0>(v, a[8 * h], a[8 * h + 1], sc);
          v = fp4_pair<1>(v, a[8 * h + 2], a[8 * h + 3], sc);
          v = fp4_pair<2>(v, a[8 * h + 4], a[8 * h + 5], sc);
          v = fp4_pair<3>(v, a[8 * h + 6], a[8 * h + 7], sc);
          p[h] = v;
        }
        // lanes below 32 end with columns 0 .. 15 of the block (their own and their
        // partner's 16 bits of two q each), the others with 16 .. 31 of the same row
        const uint2 c = swap_halves(p[0], p[1]);
        if constexpr (i == 0) wait_vmcnt<0>();  // see front(): loads that the next step reads
        const int rt = rb + l32;
        if (rt < mvalid && col < f) {
          const int64_t row = row0 + rt;
          const int fq = (f + 31) / 32 * 16, b = col / 32, nb = (f + 31) / 32;
          *reinterpret_cast<uint2*>(g.act_q + row * fq + col / 2 + 8 * lh) =
              make_uint2((c.x & 0xffffu) | (c.y << 16), (c.x >> 16) | (c.y & 0xffff0000u));
          if (lh == 0) {
            uint8_t* s = g.act_s + (static_cast<int64_t>(b >> 3) * g.cap + row) * 8;
            s[mx_pos(b)] = static_cast<uint8_t>(e8);
            if (b == nb - 1)  // the rest of the last eight, whose values are zeros
              for (int z = b + 1; (z & 7) != 0; ++z) s[mx_pos(z)] = 0;
          }
        }
      } else {
        // through the wave's patch, 16 rows of 64 columns at a time, so that
        // every store moves 16 bytes a lane and 8 lanes a whole 128-byte piece;
        // 16-byte chunk c of row r at c ^ ((r / 2) % 8)
        lds_char* const patch = ring + G::PATCHES + w * G::PATCH;
        typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));
        typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
        static_for<2>([&](auto H) {
          constexpr int h = H;
          if ((l32 >> 4) == h) {
            const int r = l32 & 15;
            static_for<2>([&](auto J) {
              static_for<4>([&](auto Q) {
                constexpr int j = J, q = Q;
                const uint2 v = pack4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2],
                                      acc[i][j][4 * q + 3]);
                *(__attribute__((address_space(3))) u32x2v*)(patch + r * 128 +
                                                             (((4 * j + q) ^ ((r >> 1) & 7)) << 4) + lh * 8) =
                    u32x2v{v.x, v.y};
              });
            });
          }
          asm volatile("" ::: "memory");
          u32x4v v[2];
          static_for<2>([&](auto Tt) {
            constexpr int t = Tt;
            const int r = 8 * t + (lane >> 3), c = lane & 7;
            v[t] = *(__attribute__((address_space(3))) u32x4v*)(patch + r * 128 + ((c ^ ((r >> 1) & 7)) << 4));
          });
          asm volatile("" ::: "memory");
          if constexpr (i == 0 && h == 0) wait_vmcnt<0>();  // see front()
          static_for<2>([&](auto Tt) {
            constexpr int t = Tt;
            const int r = 8 * t + (lane >> 3), c = lane & 7;
            const int rt = rb + 16 * h + r, col = tl.n0 + wn * 64 + 8 * c;
            if (rt < mvalid && col < d) {
              uint16_t* const to = g.y + (row0 + rt) * d + col;
              const uint4 o = make_uint4(v[t][0], v[t][1], v[t][2], v[t][3]);
              if ((d & 63) == 0) store_perm<true>(to, o);
              else store_perm<false>(to, o);
            }
          });
        });
      }
    });
  };

  // -------------------------------------------------------- tile stream
  load_tile();  // step 0 into slot 0, step 1 into slot 1
  MxTile tc = pop();
  load_a(0);
  load_b(0);
  load_s(0);
  ++lstep;
  wait_vmcnt<0>();
  if (nk == 1) load_tile();
  load_a(1);
  load_b(1);
  load_s(1);
  ++lstep;
  wait_vmcnt<0>();  // (step 1 too: a tile's first step waits for no loads)
  lgkm_drained();
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);

  Scales sc, sn;
  int slot = 0;
  auto nothing = []() {};
  while (true) {
    // Sub-steps 0 to 2 of the step in `slot`.  B's fragments of all four are read
    // in sub-step 0 and a barrier then frees B's slot, so that B (the weights,
    // which come from further away) is loaded one step and a half ahead of its
    // use where A is one; A's and B's loads thus go out half a step apart.  At the
    // end every wave has read A's slot, and the next step's values have landed:
    // all loads but the six of B and the scales that this step issued.  FIRST:
    // the tile's first step, whose next step was loaded before the epilogue's
    // stores and waited for there, so that its end does not wait for the stores.
    auto front = [&](auto AIC, auto FIRST) __attribute__((always_inline)) {
      mma_read(sc, slot, std::integral_constant<int, 0>{}, AIC, FIRST, nothing);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      mma_read(sc, slot, std::integral_constant<int, 1>{}, AIC, std::false_type{}, [&]() __attribute__((always_inline)) {
        load_b(slot);
        load_s(slot);
      });
      mma_read(sc, slot, std::integral_constant<int, 2>{}, AIC, std::false_type{}, nothing);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this wave's reads of the slot are done
      if constexpr (!FIRST) wait_vmcnt<6>();              // and the next step has landed
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
    };
    // Sub-step 3, from registers, with the next step's first fragments and A's
    // loads into the slot just read.  LAST: before the epilogue.
    auto back = [&](auto AIC, auto LAST) __attribute__((always_inline)) {
      constexpr int AI = AIC;
      lgkm_drained();
      if constexpr (!LAST) {
        load_scales(sn, slot ^ 1, AIC);
        load_first(slot ^ 1, AIC);
      }
      __builtin_amdgcn_sched_barrier(0);
      static_for<2 * AI>([&](auto T) {
        mma1(sc, std::integral_constant<int, 3>{}, T, std::false_type{});
        if constexpr (T == 0) {
          load_a(slot);
          __builtin_amdgcn_sched_barrier(0);
        }
      });
      ++lstep;
      lgkm_drained();
      __builtin_amdgcn_sched_barrier(0);
      sc = sn;
      slot ^= 1;
    };
    using T_ = std::true_type;
    using F_ = std::false_type;
    auto k_loop = [&](auto AIC) __attribute__((always_inline)) {
      fl = opaque(threadIdx.x & 63);
      lgkm_drained();
      load_scales(sc, slot, AIC);
      load_first(slot, AIC);
      // the loads are two steps ahead: from step nk - 2 on they are the next
      // tile's (or, of tiles of one step, always another's)
      if (nk <= 2) load_tile();
      front(AIC, T_{});
      if (nk > 1) {
        back(AIC, F_{});
        if (nk > 2) {
          for (int ks = 1; ks + 2 < nk; ++ks) {
            front(AIC, F_{});
            back(AIC, F_{});
          }
          static_for<AIC>([&](auto I) {
            pin(acc[I][0]);
            pin(acc[I][1]);
          });
          load_tile();
          front(AIC, F_{});
          back(AIC, F_{});
        }
        front(AIC, F_{});
      }
      back(AIC, T_{});
    };
    const int ai = wm == 0 ? (tc.h + 1) >> 1 : tc.h >> 1;
    arow0 = wm == 0 ? 0 : 32 * ((tc.h + 1) >> 1);
    static_for<AIM>([&](auto I) {
      if (ai == I + 1) k_loop(std::integral_constant<int, I + 1>{});
    });
    epilogue(tc, ai);
    tc = pop();
    if (!tc.valid) break;
  }
  wait_vmcnt<0>();
}

}  // namespace gemm
}  // namespace moe
