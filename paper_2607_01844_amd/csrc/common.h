// Internal helpers shared by the HIP kernels of the MoE library (gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#include "moe.h"

namespace moe {

constexpr int kWave = 64;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------ bf16 helpers
__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ float bf16_to_f32(uint16_t v) {
  return __uint_as_float(static_cast<uint32_t>(v) << 16);
}

// fp32 -> bf16, round to nearest even, NaN -> quiet NaN: gfx950's packed
// convert (v_cvt_pk_bf16_f32).  It agrees bit for bit with the integer
// rounding (u + 0x7fff + ((u >> 16) & 1)) >> 16 on every finite input, and
// with (u >> 16) | 0x40 on NaN (checked over all 2^32 fp32 patterns).
typedef __bf16 bf16x2_hw __attribute__((ext_vector_type(2)));
typedef float f32x2_hw __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_hw{lo, hi}, bf16x2_hw));
}
__device__ __forceinline__ uint32_t f32_to_bf16_bits(float f) { return pack_bf16x2(f, 0.0f) & 0xffffu; }
// Eight of them, two a word.
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

// Loads and stores of data that no cache needs to keep (streams far larger than
// them).  With it a copy of 2 GiB moves 5.8 TB/s instead of 5.6, and reads in
// contiguous pieces 7.1 instead of 6.2.
template <typename T>
__device__ __forceinline__ T load_stream(const T* p) {
  if constexpr (sizeof(T) == 16) {
    typedef uint32_t v4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(T, __builtin_nontemporal_load(reinterpret_cast<const v4*>(p)));
  } else if constexpr (sizeof(T) == 8) {
    typedef uint32_t v2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(T, __builtin_nontemporal_load(reinterpret_cast<const v2*>(p)));
  } else {
    return __builtin_nontemporal_load(p);
  }
}
template <typename T>
__device__ __forceinline__ void store_stream(T* p, const T& v) {
  if constexpr (sizeof(T) == 16) {
    typedef uint32_t v4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(__builtin_bit_cast(v4, v), reinterpret_cast<v4*>(p));
  } else if constexpr (sizeof(T) == 8) {
    typedef uint32_t v2 __attribute__((ext_vector_type(2)));
    __builtin_nontemporal_store(__builtin_bit_cast(v2, v), reinterpret_cast<v2*>(p));
  } else {
    __builtin_nontemporal_store(v, p);
  }
}

// ------------------------------------------------------------ wave helpers
__device__ __forceinline__ int lane_id() { return __lane_id(); }

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

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
// Compile-time loop: f(std::integral_constant<int, 0..N-1>) (keeps register
// arrays indexed by constants, so they never fall back to scratch memory).
template <typename F, int... Is>
__device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, Is...>) {
  (f(std::integral_constant<int, Is>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  static_for_impl(f, std::make_integer_sequence<int, N>{});
}

// ------------------------------------------------------------ math helpers
__device__ __forceinline__ float sigmoidf_fast(float z) { return 1.0f / (1.0f + __expf(-z)); }

// --------------------------------------------------------- launch plumbing
struct LaunchCtx {
  hipStream_t stream;
};

// Kernel ids for the optional profiler (order = moe_profile_kernel_name).
enum KernelId {
  K_ROUTE_LOGITS = 0,
  K_ROUTE_TOPK,
  K_PERM_COUNT,
  K_PERM_SCAN,
  K_PERM_RANK,
  K_PERM_GATHER,
  K_GEMM_SCHED,
  K_GEMM_FWD_GATE_UP,
  K_GEMM_FWD_DOWN,
  K_GEMM_DGRAD_DOWN,
  K_GEMM_DGRAD_GATE_UP,
  K_GEMM_WGRAD_GATE_UP,
  K_GEMM_WGRAD_DOWN,
  K_COMBINE,
  K_COMBINE_BWD,
  K_ROUTE_DLOGITS,
  K_ROUTE_DW,
  K_ROUTE_DX,
  K_VOC_LSE,
  K_VOC_GRAD,
  K_LLEP_PLAN,
  K_LLEP_WINDOW,
  K_ROUTE_SPLIT,
  K_VOC_LOGITS,
  K_VOC_DX,
  K_VOC_DW,
  K_BALANCE_PART,
  K_BALANCE_SUM,
  K_BALANCE_BWD,
  K_VOC_TEACHER,
  K_MX_QUANT,
  K_MX_GATE_UP,
  K_MX_DOWN,
  K_EMBED,
  K_EMBED_SORT,
  K_EMBED_SUM,
  K_NORM_FWD,
  K_NORM_BWD,
  K_NORM_SUM,
  K_GRAD_SUMSQ,
  K_ADAMW,
  K_ADAMW_STATES,
  K_NUM
};

// Profiler hooks (no-ops unless moe_profile_enable(1) was called).
void prof_begin(int id, hipStream_t s);
void prof_end(int id, hipStream_t s);

// Compute units of the current device (cached per device; 256 if the
// query fails).
int device_cus();

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// ------------------------------------------------------ kernel launchers
// (defined next to their kernels; arguments were validated by the C ABI)
hipError_t launch_route(const uint16_t* x, const float* w, const float* bias, int64_t T, int d,
                        int E, int k, int renorm, int32_t* idx, float* gate, float* logits,
                        hipStream_t s);
int route_bwd_chunks(int64_t T, int d, int E);
size_t route_bwd_ws_bytes(int64_t T, int d, int E);
hipError_t launch_route_bwd(const uint16_t* x, const float* w, const float* logits,
                            const int32_t* idx, const float* gate, const float* dgate,
                            const float* aux, int64_t T, int d, int E, int k, int renorm,
                            float* dw, float* dbias, uint16_t* dx, int dx_accumulate,
                            float* dlogits, void* ws, hipStream_t s);
size_t balance_ws_bytes(int64_t T, int E, int G);
hipError_t launch_balance_fwd(const float* logits, const int32_t* idx, const int32_t* off,
                              const uint8_t* mask, int64_t T, int E, int k, int G, float* balance,
                              float* zloss, int32_t* counts, float* prob_sum, int32_t* n_tokens,
                              void* ws, hipStream_t s);
hipError_t launch_balance_bwd(const float* logits, const int32_t* off, const uint8_t* mask,
                              const int32_t* counts, const int32_t* n_tokens,
                              const float* dbalance, const float* dzloss, int64_t T, int E, int k,
                              int G, int accumulate, float* dlogits, hipStream_t s);
size_t vocab_fwd_ws_bytes(int64_t N, int H, int64_t V, int64_t vblock);
size_t vocab_bwd_ws_bytes(int64_t N, int H, int64_t V, int64_t vblock);
hipError_t launch_vocab_fwd(const uint16_t* x, const uint16_t* w, const int32_t* target,
                            int64_t N, int H, int64_t V, int64_t vblock, float* loss, float* lse,
                            void* ws, size_t ws_bytes, hipStream_t s);
hipError_t launch_vocab_bwd(const uint16_t* x, const uint16_t* w, const int32_t* target,
                            const float* lse, const float* dloss, int64_t N, int H, int64_t V,
                            int64_t vblock, uint16_t* dx, uint16_t* dw, void* ws, hipStream_t s);
// A teacher's top logits of every row: K slots ids, t [N][K] (an id outside
// [0, V): no slot), tlse [N] its log-sum-exp or null (then the K slots'
// probabilities sum to one).
struct Teacher {
  const int32_t* ids;
  const float* t;
  const float* tlse;
  int K;
  float tau;
};
size_t distill_fwd_ws_bytes(int64_t N, int H, int64_t V, int64_t vblock, int K);
size_t distill_bwd_ws_bytes(int64_t N, int H, int64_t V, int64_t vblock, int K);
hipError_t launch_distill_fwd(const uint16_t* x, const uint16_t* w, const Teacher& q, int64_t N,
                              int H, int64_t V, int64_t vblock, float* loss, float* lse, float* yk,
                              void* ws, size_t ws_bytes, hipStream_t s);
hipError_t launch_distill_bwd(const uint16_t* x, const uint16_t* w, const Teacher& q,
                              const float* lse, const float* yk, const float* dloss, int64_t N,
                              int H, int64_t V, int64_t vblock, uint16_t* dx, uint16_t* dw,
                              void* ws, hipStream_t s);
size_t ffn_fwd_chunked_ws_bytes(int64_t chunk, int E, int k, int E_loc, int d, int f);
size_t ffn_fwd_row_chunked_ws_bytes(int64_t T, int E, int k, int E_loc, int d, int f,
                                    int64_t chunk_rows);
hipError_t launch_ffn_fwd_row_chunked(const uint16_t* x, const int32_t* idx, const float* gate,
                                      int64_t T, int d, int E, int k, int e_begin, int E_loc,
                                      int f, const uint16_t* wg, const uint16_t* wu,
                                      const uint16_t* wd, int64_t chunk_rows, uint16_t* y,
                                      void* ws, hipStream_t s0, hipStream_t s1);
hipError_t launch_ffn_fwd_chunked(const uint16_t* x, const int32_t* idx, const float* gate,
                                  int64_t T, int d, int E, int k, int e_begin, int E_loc, int f,
                                  const uint16_t* wg, const uint16_t* wu, const uint16_t* wd,
                                  int64_t chunk, uint16_t* y, void* ws, hipStream_t s0,
                                  hipStream_t s1);
size_t permute_ws_bytes(int64_t T, int E, int k, int E_loc);
hipError_t launch_permute(const uint16_t* x, const int32_t* idx, int64_t T, int d, int E, int k,
                          int e_begin, int E_loc, int32_t* offsets, int32_t* counts_global,
                          int32_t* row_src, int32_t* dst, uint16_t* x_perm, void* ws,
                          hipStream_t s);
hipError_t launch_gather(const uint16_t* x, const int32_t* dst, int64_t T, int d, int k,
                         uint16_t* x_perm, hipStream_t s);
// Rows [r0, r0 + rc) of a permutation (offsets, row_src over all local
// experts) as a chunk: offsets_c [E_loc + 1] relative to r0 and clamped to
// [0, rc], and x_perm_c [rc][d] (its filled rows) gathered from x.
hipError_t launch_chunk_rows(const uint16_t* x, const int32_t* row_src, const int32_t* offsets,
                             int E_loc, int64_t r0, int64_t rc, int d, int k, int32_t* offsets_c,
                             uint16_t* x_perm_c, hipStream_t s);
// launch_permute with the library's static scratch as the workspace
// (permute_ws_bytes(T, E, k, E_loc) <= MOE_PERMUTE_NOALLOC_MAX_BYTES, checked
// by the caller)
hipError_t launch_permute_noalloc(const uint16_t* x, const int32_t* idx, int64_t T, int d, int E,
                                  int k, int e_begin, int E_loc, int32_t* offsets,
                                  int32_t* counts_global, int32_t* row_src, int32_t* dst,
                                  uint16_t* x_perm, hipStream_t s);
hipError_t launch_llep_plan(const int32_t* counts, int E, int E_p, int capacity, int granule,
                            int32_t* lo, int32_t* hi, int32_t* load, int32_t* n_ship, hipStream_t s);
hipError_t launch_llep_dispatch(const uint16_t* x, const int32_t* idx, const int32_t* offsets_all,
                                const int32_t* dst_all, const int32_t* lo, const int32_t* hi,
                                int64_t T, int d, int E, int k, int64_t cap, int32_t* offsets_r,
                                int32_t* row_src_r, int32_t* dst_r, uint16_t* x_perm_r,
                                hipStream_t s);
hipError_t launch_combine(const uint16_t* y, const int32_t* dst, const float* gate, int64_t T,
                          int d, int k, uint16_t* out, hipStream_t s);
hipError_t launch_combine_bwd(const uint16_t* dout, const uint16_t* y, const int32_t* dst,
                              const float* gate, int64_t T, int d, int k, uint16_t* dy_perm,
                              float* dgate, hipStream_t s);
size_t gemm_ws_bytes(int64_t cap, int E_loc, int d, int f, unsigned flags);
// Dense products on the grouped GEMM kernel (bf16 operands, fp32 accumulation).
// Router backward, fp32 operands split as bf16 hi + lo: dl3 [T][ld3] holds
// [hi | hi | lo] of the logit gradients (E columns each), w3 [3E][d] holds
// [hi; lo; hi] of W_r^T.
//   part[c][j][e] = sum over tokens t of chunk c of x[t][j] (hi + lo)[t][e]
//   dx[t][j] = bf16([float(dx[t][j]) +] sum over the 3E columns of dl3 w3)
hipError_t launch_router_dw_mfma(const uint16_t* x, const uint16_t* dl3, int64_t T, int d, int E,
                                 int64_t ld3, int64_t chunk, float* part, hipStream_t s);
hipError_t launch_router_dx_mfma(const uint16_t* dl3, const uint16_t* w3, int64_t T, int d, int E,
                                 int64_t ld3, int accumulate, uint16_t* dx, hipStream_t s);
// Vocabulary block [v0, v0 + vb) of W [H][ldw] (B read from column bc0):
//   logits: part[n][c / 64] = (max, sum exp(y - max)) over the block's
//     columns c..c+63 of row n, yt[n] = y[n][target[n] - v0] where the
//     target lies in the block;
//   grad: G[n][c] = bf16(dloss[n] ([v0 + c == target[n]] - exp(y - lse[n]))),
//     zeros for c in [vb, gp);
//   dx: dxa[b][n][h] (=, first) or (+=) sum over c in batch b's kspan
//     columns of G[n][c] W[h][bc0 + c];
//   dw: dw[h][cc0 + c] = bf16(sum_n x[n][h] G[n][c]), row pitch ldd (rows of
//     any alignment).
hipError_t launch_vocab_logits_mfma(const uint16_t* x, const uint16_t* w, int64_t ldw, int64_t bc0,
                                    int64_t v0, int N, int H, int vb, const int32_t* target,
                                    float* part, float* yt, hipStream_t s);
hipError_t launch_vocab_grad_mfma(const uint16_t* x, const uint16_t* w, int64_t ldw, int64_t bc0,
                                  int64_t v0, int N, int H, int vb, const int32_t* target,
                                  const float* lse, const float* dloss, uint16_t* G, int64_t gp,
                                  hipStream_t s);
//   distill: the same pairs of y / tau, and yk[n][s] = y[n][ids[n][s]] for
//     slots in the block (hits: see GemmArgs); G[n][c] = bf16(coef[n]
//     exp(y / tau - lse[n])), zeros for c in [vb, gp), and, with low, `low`
//     elements on the bf16 of what that rounding left.
hipError_t launch_distill_logits_mfma(const uint16_t* x, const uint16_t* w, int64_t ldw,
                                      int64_t bc0, int64_t v0, int N, int H, int vb, float it,
                                      const uint32_t* hits, int hw, const int32_t* ids, int K,
                                      int Kp, float* part, float* yk, hipStream_t s);
hipError_t launch_distill_grad_mfma(const uint16_t* x, const uint16_t* w, int64_t ldw, int64_t bc0,
                                    int N, int H, int vb, float it, const float* lse,
                                    const float* coef, uint16_t* G, int64_t gp, int64_t low,
                                    hipStream_t s);
hipError_t launch_vocab_dx_mfma(const uint16_t* G, int64_t gp, const uint16_t* w, int64_t ldw,
                                int64_t bc0, int N, int H, int vb, int kspan, int first,
                                float* dxa, hipStream_t s);
hipError_t launch_vocab_dw_mfma(const uint16_t* x, const uint16_t* G, int64_t gp, int N, int H,
                                int vb, uint16_t* dw, int64_t ldd, int64_t cc0, hipStream_t s);
// Tile tables of the grouped products (see gemm_sched_kernel), [E_loc + 1] each.
hipError_t launch_gemm_sched(const int32_t* offsets, int E_loc, int rows, int krows,
                             int32_t* mt_start, int32_t* wk_start, int32_t* nz_start, hipStream_t s);
// MXFP4: src [B][R][C] bf16 along C (or, transpose, along R) to values q and
// scales s; back to bf16 [B][rows][K]; the grouped forward on quantised rows
// (w*[0..2]: gate, up, down); and the layer's from x and its routing.
hipError_t launch_mx_quantize(const uint16_t* src, int64_t B, int64_t R, int64_t C, int transpose,
                              uint8_t* q, uint8_t* s, hipStream_t st);
hipError_t launch_mx_dequantize(const uint8_t* q, const uint8_t* s, int64_t B, int64_t rows,
                                int64_t K, uint16_t* dst, hipStream_t st);
size_t mx_ffn_ws_bytes(int64_t cap, int E_loc, int d, int f, bool indirect);
hipError_t launch_mx_ffn(const uint8_t* xq, const uint8_t* xs, int64_t x_rows,
                         const int32_t* row_src, int k, const int32_t* offsets, int E_loc,
                         int64_t cap, int d, int f, const uint8_t* const wq[3],
                         const uint8_t* const wsc[3], uint16_t* y, void* ws, hipStream_t s);
size_t mx_layer_ws_bytes(int64_t T, int E, int k, int E_loc, int d, int f);
hipError_t launch_mx_layer(const uint16_t* x, const int32_t* idx, const float* gate, int64_t T,
                           int d, int E, int k, int e_begin, int E_loc, int f,
                           const uint8_t* const wq[3], const uint8_t* const wsc[3], uint16_t* y,
                           void* ws, hipStream_t s);
// Embedding of tokens whose rows lie in [begin, begin + rows), and its gradient.
hipError_t launch_embed_fwd(const int32_t* ids, const uint16_t* w, int64_t N, int H, int64_t begin,
                            int64_t rows, float scale, uint16_t* y, hipStream_t s);
size_t embed_bwd_ws_bytes(int64_t N, int H, int64_t rows);
hipError_t launch_embed_bwd(const int32_t* ids, const uint16_t* dy, int64_t N, int H, int64_t begin,
                            int64_t rows, float scale, uint16_t* dw, void* ws, hipStream_t s);
// Layer norm of x (+ res, with the sum in h), and its gradient.
hipError_t launch_norm_fwd(const uint16_t* x, const uint16_t* res, const float* gamma,
                           const float* beta, int64_t T, int d, float eps, uint16_t* h,
                           uint16_t* y, float* mean, float* rstd, hipStream_t s);
size_t norm_bwd_ws_bytes(int64_t T, int d);
hipError_t launch_norm_bwd(const uint16_t* dy, const uint16_t* h, const float* gamma,
                           const float* mean, const float* rstd, const uint16_t* dh, int64_t T,
                           int d, uint16_t* dx, float* dgamma, float* dbeta, void* ws,
                           hipStream_t s);
// Lists of tensors: the gradients' sum of squares, an AdamW step, and 8-bit
// states as values.
size_t grad_sumsq_ws_bytes(const moe_param* params, int count);
hipError_t launch_grad_sumsq(const moe_param* params, int count, float* sumsq, void* ws,
                             hipStream_t s);
hipError_t launch_adamw(const moe_param* params, int count, int bits, const moe_adamw_options& opt,
                        hipStream_t s);
hipError_t launch_adamw_states(const moe_param* params, int count, float* const* m, float* const* v,
                               hipStream_t s);
hipError_t launch_ffn_fwd(const uint16_t* x_perm, const int32_t* offsets, int E_loc, int64_t cap,
                          int d, int f, const uint16_t* wg, const uint16_t* wu,
                          const uint16_t* wd, uint16_t* hg, uint16_t* hu, uint16_t* y,
                          void* ws, hipStream_t s);
hipError_t launch_ffn_bwd(const uint16_t* dy, const uint16_t* x_perm, const uint16_t* hg,
                          const uint16_t* hu, const int32_t* offsets, int E_loc, int64_t cap,
                          int d, int f, const uint16_t* wg, const uint16_t* wu,
                          const uint16_t* wd, uint16_t* dx, uint16_t* dwg, uint16_t* dwu,
                          uint16_t* dwd, unsigned flags, void* ws, hipStream_t s);

}  // namespace moe
