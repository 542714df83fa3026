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
//   Both operands are loaded two steps ahead of the step being computed into
// two slots each (128 KiB, and 8 KiB of scales): a third slot for the weights,
// as the bf16 kernel has, does not fit beside the scales.  One barrier a step,
// before its last sub-step: the next step's values have landed, and the slot
// just read is free for the step after it.  The loads run on their own walk
// over the tiles (Loader), so tiles follow one another without a pause in the
// stream, however short they are.
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
  static constexpr int LDS = PATCHES + NWAVE * PATCH;  // 152 KiB, or 76 KiB
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
  }
  // no branches: one in the middle of a step would let the compiler gather the
  // step's matrix instructions behind it
  __device__ __forceinline__ void values(int j, uint32_t u, int w, int lane) const {
    const uint32_t kb = static_cast<uint32_t>(j) * 128u;
    const int lc0 = (lane & 7) ^ (lane >> 4);  // chunk of loads 0 and 2; of 1 and 3 lc0 ^ 4
    const bool in[2] = {lc0 < chunks - 8 * j, (lc0 ^ 4) < chunks - 8 * j};
#pragma unroll
    for (int q = 0; q < 4; ++q) load_lds16(rs, in[q & 1] ? voff[q] + kb : OOB, u + (4 * w + q) * 1024);
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
  constexpr int WALK = DUAL ? FWD_GATE_UP : FWD_DOWN;  // the bf16 products' tiles
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

  Tables<S> tb{g.t.mt_start, g.t.offsets, g.t.wk_start, g.t.nz_start};
  tb.init(g.t.E_loc, lane);

  // ------------------------------------------------------------ loads
  TileIter<WALK, S> lit;  // the loads' walk over the tiles, ahead of the products'
  lit.init(g.t, tb);
  MxStream sa, sb;
  int lstep = nk;     // the next step to load of the loads' tile (nk: take the next tile)
  auto load_tile = [&]() __attribute__((always_inline)) {
    const Tile t = lit.next(g.t, tb);
    lstep = 0;
    if (!t.valid) {
      sa.none();
      sb.none();
      return;
    }
    {
      const int64_t r0 = static_cast<int64_t>(t.seg) + t.m0 + 32 * w;
      const int rows = min(t.ne - t.m0, 32 * t.h) - 32 * w;
      if (g.a_tok != nullptr) {
        const int32_t* tok = g.a_tok + r0;
        sa.setup(g.a.q, g.a_bytes, kq, rows, [&](int r) { return r < rows ? tok[r] : 0; }, g.a.s, g.a_rows,
                 r0, lane);
      } else {
        sa.setup(g.a.q + r0 * kq, static_cast<int64_t>(rows) * kq, kq, rows, [](int r) { return r; }, g.a.s,
                 g.a_rows, r0, lane);
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
  // part p (0: A's values, 1: B's, 2: scales) of the step `lstep` into slot `slot`
  auto load_part = [&](int slot, int p) __attribute__((always_inline)) {
    const int ln = opaque(threadIdx.x & 63);
    if (p == 0) sa.values(lstep, lds0 + slot * UNIT, w, ln);
    else if (p == 1) sb.values(lstep, lds0 + (2 + slot) * UNIT, w, ln);
    else {
      sa.scales(lstep, lds0 + G::SCALES + slot * SUNIT, w, ln);
      sb.scales(lstep, lds0 + G::SCALES + (2 + slot) * SUNIT, w, ln);
    }
  };

  // --------------------------------------------------------- products
  int arow0 = 0, brow[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) brow[j] = DUAL ? j * (S / 2) + wn * 32 : wn * 64 + 32 * j;
  f32x16 acc[AIM][2];
  auto zero_acc = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < AIM; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  };
  struct Frags {
    i32x4v a[AIM], b[2];
  };
  struct Scales {
    int a[AIM], b[2];
  };
  int fl = lane;  // the lane, made opaque tile by tile: addresses of one row-block
                  // count are not kept live through another's loop
  // fragment f (0 .. AIM - 1: A's row blocks, then B's two) of sub-step `sub`
  auto load_frag1 = [&](Frags& F, int slot, int sub, auto FI) __attribute__((always_inline)) {
    constexpr int fi = FI;
    if constexpr (fi < AIM) {
      const lds_char* t = ring + slot * UNIT + (arow0 + 32 * fi) * 128;
      F.a[fi] = *reinterpret_cast<const __attribute__((address_space(3))) i32x4v*>(t + koff(fl & 31, 2 * sub + (fl >> 5)));
    } else {
      const lds_char* t = ring + (2 + slot) * UNIT + brow[fi - AIM] * 128;
      F.b[fi - AIM] = *reinterpret_cast<const __attribute__((address_space(3))) i32x4v*>(t + koff(fl & 31, 2 * sub + (fl >> 5)));
    }
  };
  auto load_frags = [&](Frags& F, int slot, int sub, auto AIC) __attribute__((always_inline)) {
    static_for<AIM + 2>([&](auto FI) {
      if constexpr (FI >= AIM || FI < AIC) load_frag1(F, slot, sub, FI);
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
  auto mma1 = [&](const Frags& F, const Scales& c, auto SUB, auto T) __attribute__((always_inline)) {
    constexpr int i = T / 2, j = T % 2;
    const i32x8 bv = __builtin_shufflevector(F.b[j], F.b[j], 0, 1, 2, 3, -1, -1, -1, -1);
    const i32x8 av = __builtin_shufflevector(F.a[i], F.a[i], 0, 1, 2, 3, -1, -1, -1, -1);
    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(bv, av, acc[i][j], 4, 4, SUB, c.b[j], SUB, c.a[i]);
  };
  // the 2 AI products of sub-step SUB, with the next sub-step's fragment reads
  // between them in the order that its products need them
  auto mma_read = [&](const Frags& F, Frags& Gn, const Scales& c, int slot, auto SUB, auto AIC)
      __attribute__((always_inline)) {
    constexpr int AI = AIC, per = AI == 1 ? 2 : 1;
    static_for<2 * AI>([&](auto T) {
      mma1(F, c, SUB, T);
      __builtin_amdgcn_sched_barrier(0);
      static_for<per>([&](auto P) {
        constexpr int r = per * T + P;
        if constexpr (r < AI + 2) {
          constexpr int f0 = r == 0 ? 0 : r == 1 ? AIM : r == 2 ? AIM + 1 : r - 2;
          load_frag1(Gn, slot, SUB + 1, std::integral_constant<int, f0>{});
          __builtin_amdgcn_sched_barrier(0);
        }
      });
    });
  };

  // --------------------------------------------------------- epilogue
  // acc[i][j][4 q + u]: output row arow0 + 32 i + l32, column brow[j] + 8 q + 4 lh + u
  auto epilogue = [&](const Tile& tl, int ai) __attribute__((always_inline)) {
    const int mvalid = min(tl.ne - tl.m0, 32 * tl.h);
    const int64_t row0 = static_cast<int64_t>(tl.seg) + tl.m0;
    // lane-derived indices formed here, not kept live across the K loop
    const int lane = opaque(threadIdx.x & 63), l32 = lane & 31, lh = lane >> 5;
    static_for<AIM>([&](auto I) {
      constexpr int i = I;
      if (i >= ai) return;
      const int rb = arow0 + 32 * i;
      if (rb >= mvalid) return;
      if constexpr (DUAL) {
        // The wave's 32 columns of a row are one block of the down product's
        // contraction: lanes l and l + 32 hold 16 each.
        const int col = tl.n0 + wn * 32;
        if (col >= f) return;
        float a[16];
        uint32_t top = 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float z = acc[i][0][r];
          a[r] = z * sigmoidf_fast(z) * acc[i][1][r];
          top = max(top, __float_as_uint(a[r]) & 0x7fffffffu);
        }
        top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 32, 64)));
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
        const uint32_t o0 = static_cast<uint32_t>(__shfl_xor(static_cast<int>(p[0]), 32, 64));
        const uint32_t o1 = static_cast<uint32_t>(__shfl_xor(static_cast<int>(p[1]), 32, 64));
        const int rt = rb + l32;
        if (lh == 0 && rt < mvalid) {
          const int64_t row = row0 + rt;
          const int fq = (f + 31) / 32 * 16, b = col / 32, nb = (f + 31) / 32;
          *reinterpret_cast<uint4*>(g.act_q + row * fq + col / 2) =
              make_uint4((p[0] & 0xffffu) | (o0 << 16), (p[0] >> 16) | (o0 & 0xffff0000u),
                         (p[1] & 0xffffu) | (o1 << 16), (p[1] >> 16) | (o1 & 0xffff0000u));
          uint8_t* s = g.act_s + (static_cast<int64_t>(b >> 3) * g.cap + row) * 8;
          s[mx_pos(b)] = static_cast<uint8_t>(e8);
          if (b == nb - 1)  // the rest of the last eight, whose values are zeros
            for (int c = b + 1; (c & 7) != 0; ++c) s[mx_pos(c)] = 0;
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
          static_for<2>([&](auto Tt) {
            constexpr int t = Tt;
            const int r = 8 * t + (lane >> 3), c = lane & 7;
            const u32x4v v = *(__attribute__((address_space(3))) u32x4v*)(patch + r * 128 +
                                                                          ((c ^ ((r >> 1) & 7)) << 4));
            const int rt = rb + 16 * h + r, col = tl.n0 + wn * 64 + 8 * c;
            if (rt < mvalid && col < d) {
              uint16_t* const to = g.y + (row0 + rt) * d + col;
              if ((d & 63) == 0) store_perm<true>(to, make_uint4(v[0], v[1], v[2], v[3]));
              else store_perm<false>(to, make_uint4(v[0], v[1], v[2], v[3]));
            }
          });
          asm volatile("" ::: "memory");
        });
      }
    });
  };

  // -------------------------------------------------------- tile stream
  TileIter<WALK, S> it;
  it.init(g.t, tb);
  Tile tc = it.next(g.t, tb);
  if (!tc.valid) return;
  // step 0 into slot 0, step 1 into slot 1
  auto load_step = [&](int slot) __attribute__((always_inline)) {
    if (lstep == nk) load_tile();
    load_part(slot, 0);
    load_part(slot, 1);
    load_part(slot, 2);
    ++lstep;
  };
  load_step(0);
  wait_vmcnt<0>();
  load_step(1);
  lgkm_drained();
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);

  Frags cur, nxt;
  Scales sc, sn;
  int slot = 0;
  zero_acc();
  while (true) {
    auto step = [&](auto AIC) __attribute__((always_inline)) {
      constexpr int AI = AIC;
      if (lstep == nk) load_tile();
      mma_read(cur, nxt, sc, slot, std::integral_constant<int, 0>{}, AIC);
      mma_read(nxt, cur, sc, slot, std::integral_constant<int, 1>{}, AIC);
      mma_read(cur, nxt, sc, slot, std::integral_constant<int, 2>{}, AIC);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this wave's reads of the slot are done
      wait_vmcnt<0>();                                    // and the next step has landed
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      lgkm_drained();
      load_scales(sn, slot ^ 1, AIC);
      load_frags(cur, slot ^ 1, 0, AIC);
      __builtin_amdgcn_sched_barrier(0);
      static_for<2 * AI>([&](auto T) {
        constexpr int t = T;
        mma1(nxt, sc, std::integral_constant<int, 3>{}, T);
        __builtin_amdgcn_sched_barrier(0);
        static_for<3>([&](auto P) {
          constexpr int p = P;
          if constexpr (p * 2 * AI / 3 == t) {
            load_part(slot, p);
            __builtin_amdgcn_sched_barrier(0);
          }
        });
      });
      ++lstep;
      lgkm_drained();
      __builtin_amdgcn_sched_barrier(0);
      sc = sn;
      slot ^= 1;
    };
    auto k_loop = [&](auto AIC) __attribute__((always_inline)) {
      fl = opaque(threadIdx.x & 63);
      lgkm_drained();
      load_scales(sc, slot, AIC);
      load_frags(cur, slot, 0, AIC);
      for (int ks = 0; ks < nk; ++ks) step(AIC);
    };
    const int ai = wm == 0 ? (tc.h + 1) >> 1 : tc.h >> 1;
    arow0 = wm == 0 ? 0 : 32 * ((tc.h + 1) >> 1);
    static_for<AIM>([&](auto I) {
      if (ai == I + 1) k_loop(std::integral_constant<int, I + 1>{});
    });
    epilogue(tc, ai);
    tc = it.next(g.t, tb);
    if (!tc.valid) break;
    zero_acc();
  }
  wait_vmcnt<0>();
}

}  // namespace gemm
}  // namespace moe
