// octo_op_product: rows times weights with bias, activation or gate, and residual.
//
//   y[i][j] = act(sum_k x[i][k] w[j][k] + b[j]) + r[i][j],     gated: act(z[i][j]) z[i][cols + j] + r[i][j], z the sums of all 2 cols rows of w
//
// Rows of w and of x are alike: both are read along k, 16 bytes a lane, and go into the matrix instructions as they lie in memory.  w is the first operand, so a lane gets
// results of neighbouring outputs of one token.
//
// Measured (MI355X): 8192 cubed bf16 1447 TFLOP/s (a large library product 1580), 8 bits 1451 (with fast8 2540), fp32 144; 12800 tokens 4096 -> 4096 bf16 318 us; 512 tokens of it 22; 16 tokens 4096 -> 131072
// bf16 184 us, 5.8 TB/s; 16 tokens 4096 -> 2 x 12288 in 8 bits, gated, 24 us and to 8 bits 28, 4.2 and 3.6 TB/s.
#pragma once
#include <utility>

#include "mx8.h"
#include "octo_internal.h"
#include "product_choice.h"

namespace octo {

enum { PRODUCT_Y_F32 = 0, PRODUCT_Y_F16 = 1, PRODUCT_Y_BF16 = 2, PRODUCT_Y_MX8 = 3 };
enum { PRODUCT_ACT_NONE = 0, PRODUCT_ACT_RELU = 1, PRODUCT_ACT_SILU = 2, PRODUCT_ACT_GELU = 3 };

struct ProductArgs {
  const char* x; const char* w;                       // rows of k_bytes, x_row and w_row bytes apart
  const uint8_t* xe; const uint8_t* we;               // exponents of rows in 8 bits
  long long x_row, w_row, xe_row, we_row;
  const float* bias; const void* res; void* y;
  long long res_row, y_row;                           // in elements
  octo_mx8_rows y8;
  const int* n_dyn;
  int n, k_bytes, cols, gated, act, y_kind;
  int y_vec, res_vec, bias_vec;                       // four values at a multiple of four outputs are one aligned vector
  int vec;                                            // all of them are (or are not there), and outputs are whole vectors, not in 8 bits
  int exp_words;                                      // the exponents of 128 values of k are one aligned word
  int exact8;                                         // rows of 8 bits go through bf16 also where tokens are many: sums in fp32
  int direct;                                         // results of 16 bits, eight of them one aligned vector, or of 8 bits, activations that take few instructions
  int tiles_n, tiles_m;
  int n_from;                                         // tokens before x's first row, of those that n_dyn counts
};

__device__ __forceinline__ int product_tokens(const ProductArgs& a) { return a.n_dyn ? min(max(max(*a.n_dyn, 0) - a.n_from, 0), a.n) : a.n; }

typedef __attribute__((address_space(3))) unsigned char LdsBytes;

__device__ __forceinline__ float relu(float v) { return v < 0.f ? 0.f : v; }      // NaN stays (fmaxf would take the other one)
__device__ __forceinline__ float product_act(int act, float v) {
  if (act == PRODUCT_ACT_RELU) return relu(v);
  if (act == PRODUCT_ACT_SILU) return silu(v);
  if (act == PRODUCT_ACT_GELU) return 0.5f * v * erfcf(v * -0.70710678118654752f);      // 1 + erf cancels: at v = -4.5 a twentieth is wrong, below -5.5 all of it
  return v;
}

template <typename T> __device__ __forceinline__ void product_read4(const void* p, long long at, int have, int vec, float* v) {
  const T* r = (const T*)p + at;
  if (vec && have == 4) {
    const floatx4 f = load4(r);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += f[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) if (e < have) v[e] += (float)r[e];
  }
}
template <typename T> __device__ __forceinline__ void product_write4(void* p, long long at, int have, int vec, const float* v) {
  T* y = (T*)p + at;
  if (vec && have == 4) {
    store4<T>(y, floatx4{v[0], v[1], v[2], v[3]});
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) if (e < have) y[e] = (T)v[e];
  }
}

// The sums of outputs j .. j + 3 (a multiple of four) of token i become results: z, and up where the layer is gated.  Where they go to 8 bits, the eight lanes of a group of 32
// outputs call it together.  `on`: the token is there.
__device__ __forceinline__ void product_finish4(const ProductArgs& a, bool on, int i, int j, floatx4 z, floatx4 up) {
  const int have = min(4, a.cols - j);
  on = on && have > 0;
  float v[4] = {z[0], z[1], z[2], z[3]};
  if (a.bias && on) product_read4<float>(a.bias, j, have, a.bias_vec, v);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = product_act(a.act, v[e]);
  if (a.gated) {
    float u[4] = {up[0], up[1], up[2], up[3]};
    if (a.bias && on) product_read4<float>(a.bias, (long long)a.cols + j, have, a.bias_vec, u);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= u[e];
  }
  if (a.y_kind == PRODUCT_Y_MX8) {
    unsigned most = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) most = max(most, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    if (!on) most = 0;
#pragma unroll
    for (int d = 1; d < 8; d *= 2) most = max(most, (unsigned)__shfl_xor((int)most, d));
    if (!on) return;
    const bool none = most >= 0x7F800000u;
    const int ex = mx8_exp(most);
    *(unsigned*)(a.y8.d_codes + i * a.y8.code_row + j) = none ? MX8_NAN4 : mx8_pack4(floatx4{v[0], v[1], v[2], v[3]}, mx8_inverse(ex));
    if (j % 32 == 0) a.y8.d_exps[i * a.y8.exp_row + j / 32] = (uint8_t)(none ? 255 : ex);
    return;
  }
  if (!on) return;
  const long long ry = i * a.res_row + j, wy = i * a.y_row + j;
  if (a.y_kind == PRODUCT_Y_F32) {
    if (a.res) product_read4<float>(a.res, ry, have, a.res_vec, v);
    product_write4<float>(a.y, wy, have, a.y_vec, v);
  } else if (a.y_kind == PRODUCT_Y_F16) {
    if (a.res) product_read4<_Float16>(a.res, ry, have, a.res_vec, v);
    product_write4<_Float16>(a.y, wy, have, a.y_vec, v);
  } else {
    if (a.res) product_read4<__bf16>(a.res, ry, have, a.res_vec, v);
    product_write4<__bf16>(a.y, wy, have, a.y_vec, v);
  }
}

// The same for B pieces of four outputs at once, whose residuals and biases are in flight together.  Only where `a.vec`: all of it in aligned vectors of four.
template <typename Y, int B>
__device__ __forceinline__ void product_finish_vec(const ProductArgs& a, const bool* on, const int* i, const int* j, floatx4* z, floatx4* up) {
  floatx4 res[B];
  if (a.bias) {
    floatx4 b0[B], b1[B];
#pragma unroll
    for (int b = 0; b < B; ++b) b0[b] = on[b] ? *(const floatx4*)(a.bias + j[b]) : floatx4{0.f, 0.f, 0.f, 0.f};
    if (a.gated) {
#pragma unroll
      for (int b = 0; b < B; ++b) b1[b] = on[b] ? *(const floatx4*)(a.bias + a.cols + j[b]) : floatx4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int b = 0; b < B; ++b) { z[b] += b0[b]; if (a.gated) up[b] += b1[b]; }
  }
  if (a.res) {
#pragma unroll
    for (int b = 0; b < B; ++b) if (on[b]) res[b] = load4((const Y*)a.res + i[b] * a.res_row + j[b]);
  }
  auto act = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e) z[b][e] = f(z[b][e]);
  };
  if (a.act == PRODUCT_ACT_SILU) act([](float v) { return silu(v); });
  else if (a.act == PRODUCT_ACT_RELU) act([](float v) { return relu(v); });
  else if (a.act == PRODUCT_ACT_GELU) act([](float v) { return product_act(PRODUCT_ACT_GELU, v); });
  if (a.gated) {
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e) z[b][e] *= up[b][e];
  }
#pragma unroll
  for (int b = 0; b < B; ++b) {
    if (!on[b]) continue;
    if (a.res) {
#pragma unroll
      for (int e = 0; e < 4; ++e) z[b][e] += res[b][e];
    }
    store4((Y*)a.y + i[b] * a.y_row + j[b], z[b]);
  }
}

// Products of 16 x 16 blocks: a lane (row l % 16, part g = l / 16) gives 16 bytes of its row of each operand and gets rows 4 g .. + 3 of column l % 16.  Under the power limit these run 14 % (8
// bits: 8 %) faster than 32 x 32 blocks (bf16 registers alone 2113 TFLOP/s and 1849, 8 bits 4428 and 4096).
template <typename T>
__device__ __forceinline__ floatx4 mfma_part(u32x4 a, u32x4 b, floatx4 c) {
  if constexpr (sizeof(T) == 4) {
    const floatx4 w = __builtin_bit_cast(floatx4, a), x = __builtin_bit_cast(floatx4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], x[e], c, 0, 0, 0);
    return c;
  } else {
    return mfma16<T>(a, b, c);
  }
}
// In 8 bits, 128 values of k: bytes 16 g .. + 15 of both halves, and the exponent of block g of its row.
__device__ __forceinline__ floatx4 mfma_mx8(const u32x4* a, const u32x4* b, floatx4 c, int ea, int eb) {
  typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
  const u32x8 x = __builtin_shufflevector(a[0], a[1], 0, 1, 2, 3, 4, 5, 6, 7), y = __builtin_shufflevector(b[0], b[1], 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_bit_cast(i32x8, x), __builtin_bit_cast(i32x8, y), c, 0, 0, 0, ea, 0, eb);
}

// Eight and sixteen values of 8 bits in bf16, which holds them and their power of two exactly (codes of the bytes 1 and 2 to the next multiple of 2^-133); `e`: their exponent byte.
__device__ __forceinline__ u32x4 widen_mx8(unsigned v0, unsigned v1, unsigned e) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const float scale = __uint_as_float(e << 23);
  return u32x4{__builtin_bit_cast(unsigned, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)v0, scale, false)), __builtin_bit_cast(unsigned, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)v0, scale, true)),
               __builtin_bit_cast(unsigned, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)v1, scale, false)), __builtin_bit_cast(unsigned, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)v1, scale, true))};
}
__device__ __forceinline__ void widen_mx8(u32x4 v, unsigned e, u32x4* lo, u32x4* hi) { *lo = widen_mx8(v[0], v[1], e); *hi = widen_mx8(v[2], v[3], e); }

// A wavefront's sums, 2 TN x 2 TM blocks of 16 rows of w times 16 tokens (of a gated layer: two of gates, two of what they are gates of, ...), straight from its registers.  An
// exchange between rows of 16 lanes makes 16 bytes of neighbouring outputs a lane, 64 bytes a token of every store: the lane's chunk of eight outputs is then {0, 2, 1, 3}[g].  For
// results of 16 or 8 bits whose rows are aligned (`a.direct`).
struct DirectMx8 {};
template <typename Y, int TN, int TM, bool GATED>
__device__ __forceinline__ void finish_direct_as(const ProductArgs& a, floatx4 (&acc)[2 * TN][2 * TM], int n, int tok0, int col0, int lane) {
  constexpr bool TO8 = std::is_same<Y, DirectMx8>::value;
  constexpr int STEP = GATED ? 4 : 2;
  typedef typename std::conditional<TO8, __bf16, Y>::type Y16;
  const int g = lane >> 4, turned = (g & 1) * 2 + (g >> 1);
  auto swap = [](u32x2& x, u32x2& z) __attribute__((always_inline)) {          // its own inverse
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const auto r = __builtin_amdgcn_permlane16_swap(x[e], z[e], false, false);
      x[e] = r[0]; z[e] = r[1];
    }
  };
#pragma unroll
  for (int i = 0; i < 2 * TN; i += STEP) {
    const int col = col0 + i / STEP * 32;
    if (col >= a.cols) return;
    const int c = col + turned * 8;
    u32x4 res[2 * TM];
    if (!TO8 && a.res) {
#pragma unroll
      for (int j = 0; j < 2 * TM; ++j) {
        const int tok = tok0 + j * 16 + (lane & 15);
        res[j] = u32x4{0, 0, 0, 0};
        if (tok < n && c < a.cols) res[j] = *(const u32x4*)((const Y16*)a.res + tok * a.res_row + c);
      }
    }
    floatx4 b0[2], b1[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = col + 16 * h + 4 * g;
      b0[h] = a.bias && at < a.cols ? *(const floatx4*)(a.bias + at) : floatx4{0.f, 0.f, 0.f, 0.f};
      b1[h] = GATED && a.bias && at < a.cols ? *(const floatx4*)(a.bias + a.cols + at) : floatx4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int j = 0; j < 2 * TM; ++j) {
      // the sums of the largest tiles fill one half of the registers and are taken out of it block by block, here and not before
      if constexpr (TN * TM >= 16) {
#pragma unroll
        for (int h = 0; h < STEP; ++h) asm volatile("" : "+a"(acc[i + h][j]));
      }
      floatx4 v[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) v[h] = acc[i + h][j] + b0[h];
      auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[h][e] = f(v[h][e]);
      };
      if (a.act == PRODUCT_ACT_SILU) each([](float z) { return silu(z); });
      else if (a.act == PRODUCT_ACT_RELU) each([](float z) { return relu(z); });
      if constexpr (GATED) {
#pragma unroll
        for (int h = 0; h < 2; ++h) v[h] *= acc[i + 2 + h][j] + b1[h];
      }
      const int tok = tok0 + j * 16 + (lane & 15);
      if constexpr (TO8) {
        unsigned most = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) most = max(most, __float_as_uint(v[h][e]) & 0x7FFFFFFFu);
        most = max(most, (unsigned)__shfl_xor((int)most, 16));
        most = max(most, (unsigned)__shfl_xor((int)most, 32));
        const bool none = most >= 0x7F800000u;
        const int ex = mx8_exp(most);
        const float inverse = mx8_inverse(ex);
        const auto r = __builtin_amdgcn_permlane16_swap(none ? MX8_NAN4 : mx8_pack4(v[0], inverse), none ? MX8_NAN4 : mx8_pack4(v[1], inverse), false, false);
        if (tok < n) {
          *(u32x2*)(a.y8.d_codes + tok * a.y8.code_row + c) = u32x2{r[0], r[1]};
          if (!g) a.y8.d_exps[tok * a.y8.exp_row + col / 32] = (uint8_t)(none ? 255 : ex);
        }
      } else {
        if (a.res) {
          u32x2 x = {res[j][0], res[j][1]}, z = {res[j][2], res[j][3]};
          swap(x, z);
          v[0] += load4((const Y16*)&x);
          v[1] += load4((const Y16*)&z);
        }
        u32x2 x, z;
        store4<Y16>((Y16*)&x, v[0]);
        store4<Y16>((Y16*)&z, v[1]);
        swap(x, z);
        if (tok < n && c < a.cols) *(u32x4*)((Y16*)a.y + tok * a.y_row + c) = u32x4{x[0], x[1], z[0], z[1]};
      }
    }
  }
}
template <typename Y, int TN, int TM>
__device__ __forceinline__ void finish_direct(const ProductArgs& a, floatx4 (&acc)[2 * TN][2 * TM], int n, int tok0, int col0, int lane) {
  if (a.gated) finish_direct_as<Y, TN, TM, true>(a, acc, n, tok0, col0, lane);
  else finish_direct_as<Y, TN, TM, false>(a, acc, n, tok0, col0, lane);
}

// f(integral_constant 0), .. f(integral_constant N - 1): loops whose bodies have other loops with bounds by their counter
template <typename F, int... I> __device__ __forceinline__ void unrolled(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, typename F> __device__ __forceinline__ void unrolled(F&& f) { unrolled(f, std::make_integer_sequence<int, N>{}); }

// ---- many tokens: tiles in LDS -----------------------------------------------------------------------------------------
// A block makes BN rows of w times BM tokens; its WN x WM wavefronts take TN x TM blocks of 32 x 32 each.  A step covers 128 bytes of k of all rows.  Loads go straight
// to LDS, two steps deep: once all wavefronts have read their last operands of step t, its place is given to step t + 2, whose loads then have a whole step's products to
// arrive in.  Operands of the next products are read from LDS while the present ones run, also across steps, so a step costs one barrier in the middle of
// products.  The 16-byte chunks of a row lie at their number xor half
// the row's, which spreads the rows that sixteen lanes read together over all banks.
//
// Rows of 8 bits (EXACT): values are widened to bf16, whose products are exact and added in fp32.  The 8-bit matrix instructions are twice as fast, but add products in groups of eight at the weight
// of the group's largest and drop what lies 2^13 below it (measured: 1 + 2^-13 comes out, 1 + 2^-14 does not), 2^-14 of a sum's size in the mean, and all of it where the large ones cancel: they
// run where the caller permits it, and results are rounded to 16 or 8 bits.  (12800 tokens 4096 -> 2 x 12288, gated: 1867 us, with fast8 1070; 8192 cubed 758 and 433; 128 tokens 4096 -> 4096
// 25.6 and 16.3.)
// The size of four stages is given at the launch: a compiler that knows it, and that a CU has room for one block, lets a wavefront have both halves of the registers, and moves sums
// from one half to the other and back in each step (512 tokens, bf16 4096 -> 4096: 27.6 us, so 21.9).
template <int D, int BYTES> struct ProductLds {
  static __device__ __forceinline__ unsigned char* at() { __shared__ __attribute__((aligned(1024))) unsigned char smem[BYTES]; return smem; }
};
template <int BYTES> struct ProductLds<4, BYTES> {
  static __device__ __forceinline__ unsigned char* at() { extern __shared__ __attribute__((aligned(1024))) unsigned char product_stages[]; return product_stages; }
};
template <typename T, bool EXACT, int TN, int TM, int WN, int WM, int D> struct ProductTile {
  static constexpr bool MX = std::is_same<T, f8>::value;
  static constexpr int NW = WN * WM, BN = WN * TN * 32, BM = WM * TM * 32, ROWS = BN + BM, STAGE = ROWS * 128, LW = BN / 8 / NW, LX = BM / 8 / NW;
  static constexpr int HT = TM < 2 ? 1 : 2, UNIT = HT * 32 * TN * 32 * 4;      // sums of a wavefront on their way out, of 32 or 64 tokens
  static constexpr int NE = MX ? (ROWS + NW * 64 - 1) / (NW * 64) : 1, EXPS = NE * NW * 64;   // exponents of a step, whole loads
  static constexpr int RING = EXACT ? 4 : D, MAIN = D * STAGE + (MX ? RING * EXPS * 4 : 0), LDS = MAIN > NW * UNIT ? MAIN : NW * UNIT;
};
template <typename T, bool EXACT, int TN, int TM, int WN, int WM, int MINB, int D>
__global__ __launch_bounds__(WN * WM * 64, MINB) void product_tile_kernel(ProductArgs a) {
  using P = ProductTile<T, EXACT, TN, TM, WN, WM, D>;
  constexpr bool MX = P::MX;
  constexpr int NW = P::NW, BN = P::BN, BM = P::BM, ROWS = P::ROWS, STAGE = P::STAGE, LW = P::LW, LX = P::LX, HT = P::HT, UNIT = P::UNIT, NE = P::NE, EXPS = P::EXPS, RING = P::RING;
  constexpr int BW = 2 * TN, BX = 2 * TM, M = BW * BX, L = LW + LX;   // blocks of 16 rows of a wavefront, their products, loads of a step
  static_assert(BN / 8 % NW == 0 && BM / 8 % NW == 0 && TN % 2 == 0 && NW % 4 == 0, "whole loads a wavefront, pairs of blocks");
  using Lds = ProductLds<D, P::LDS>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
  const int wn = wave % WN, wm = wave / WN;
  const int n = product_tokens(a);

  // Tiles in groups of eight along the tokens, all outputs of a group one after the other, and an eighth of that list to each die (block b runs on die b % 8): the
  // blocks of a die share rows of w and x in its L2.
  int tn, tm;
  {
    const int tiles = a.tiles_n * a.tiles_m, die = blockIdx.x % 8, i = blockIdx.x / 8, base = tiles / 8, more = tiles % 8;
    const int id = die * base + min(die, more) + i;
    const int group = id / (8 * a.tiles_n), first = group * 8, tall = min(8, a.tiles_m - first), in = id - group * 8 * a.tiles_n;
    tm = first + in % tall; tn = in / tall;
  }
  const int m0 = tm * BM, n0 = tn * (a.gated ? BN / 2 : BN);         // the tile's first token and output
  if (m0 >= n) return;

  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(LdsBytes*)Lds::at());
  // Load q of a wavefront brings rows 8 (LW wave + q) .. + 7 of the tile (of x: LX wave + ..), 1024 bytes behind load q - 1.  The places in LDS of four loads differ by the instructions' offset
  // alone, which is taken off the addresses again: each write of m0 holds the wavefront up for some twenty cycles (16 a step: 2460 cycles for 2048 of products).
  const int row8 = lane >> 3;
  int woff[LW], xoff[LX];
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    const int row = (wave * LW + i) * 8 + row8, chunk = (lane & 7) ^ (row >> 1 & 7);
    const int col = a.gated ? row / 64 * 32 + row % 32 : row;
    woff[i] = n0 + col < a.cols ? col * (int)a.w_row + chunk * 16 + 4096 - i % 4 * 1024 : OOB;
  }
#pragma unroll
  for (int i = 0; i < LX; ++i) {
    const int row = (wave * LX + i) * 8 + row8, chunk = (lane & 7) ^ (row >> 1 & 7);
    xoff[i] = m0 + row < n ? row * (int)a.x_row + chunk * 16 + 4096 - i % 4 * 1024 : OOB;
  }
  const char* const w0 = a.w + n0 * a.w_row;
  const char* const w1 = w0 + (a.gated ? a.cols * a.w_row : 0);
  const char* const x0 = a.x + m0 * a.x_row;
  const int nk = (a.k_bytes + 127) / 128;

  // Exponents, a word for each row and step, two steps deep (EXACT: four): a thread has row threadIdx.x and those NW * 64 further on.  Whole words go straight to LDS.  Otherwise (EXACT
  // alone) bytes are taken one by one to registers, since what lies behind a row's end may read as NaN, and placed a step later.
  const uint8_t* exp_at[NE];
  unsigned exps[NE];
  if constexpr (MX) {
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const int r = i * NW * 64 + (int)threadIdx.x;
      const int col = min(n0 + (a.gated ? r / 64 * 32 + r % 32 : r), a.cols - 1), tok = min(m0 + max(r - BN, 0), n - 1);      // of a row that is not there: any row's
      exp_at[i] = r < BN ? a.we + ((a.gated && r / 32 % 2 ? (long long)a.cols : 0) + col) * a.we_row : a.xe + tok * a.xe_row;
    }
  }
  auto load_exps = [&](int t) __attribute__((always_inline)) {       // bytes
    if constexpr (MX && EXACT) {
      if (!a.exp_words) {
#pragma unroll
        for (int i = 0; i < NE; ++i) {
          exps[i] = 0;
#pragma unroll
          for (int b = 0; b < 4; ++b) if (t * 128 + b * 32 < a.k_bytes) exps[i] |= (unsigned)exp_at[i][4 * t + b] << (8 * b);
        }
      }
    }
  };
  auto place_exps = [&](int t) __attribute__((always_inline)) {
    if constexpr (MX && EXACT) {
      if (!a.exp_words) {
#pragma unroll
        for (int i = 0; i < NE; ++i) {
          const int r = i * NW * 64 + (int)threadIdx.x;
          if (r < ROWS) *(unsigned*)(Lds::at() + D * STAGE + ((t & (RING - 1)) * EXPS + r) * 4) = exps[i];
        }
      }
    }
  };
  auto issue_exps = [&](int t) __attribute__((always_inline)) {      // words
    if constexpr (MX) {
      if (!EXACT || a.exp_words) {
#pragma unroll
        for (int i = 0; i < NE; ++i)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                         :: "s"(lds + D * STAGE + ((t & (RING - 1)) * EXPS + (i * NW + wave) * 64) * 4), "v"(exp_at[i] + 4 * min(t, nk - 1)) : "memory");
      }
    }
  };
  // Lanes whose chunk of step t lies behind their row's end, of loads of even and odd number: they load nothing from there on.  (No branches in the loop: products would move across them.)
  bool gone[2];
  auto cut = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) gone[odd] = ((lane & 7) ^ (odd * 4 + (lane >> 4))) * 16 + t * 128 >= a.k_bytes;
  };
  // load q of step t: LW of w, then LX of x.  Addresses are 4096 too large, for the offsets, and buffers start as much earlier.
  auto issue = [&](int t, int stage, int q) __attribute__((always_inline)) {
    const bool is_w = q < LW;
    const int i = is_w ? q : q - LW;
    int& off = is_w ? woff[is_w ? i : 0] : xoff[is_w ? 0 : i];
    off = gone[i & 1] ? OOB : off;
    // rows of a gated layer alternate between its halves, 32 at a time
    const bool second = is_w && ((LW % 8 == 0 ? i / 4 : (wave * LW + i) / 4) & 1);
    const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc((void*)((is_w ? second ? w1 : w0 : x0) + t * 128 - 4096), 0, 0x7FFFFFFF, BUF_FLAGS);
    const unsigned to = lds + stage * STAGE + (is_w ? wave * LW * 1024 : BN * 128 + wave * LX * 1024) + i / 4 * 4096;
    if (i % 4 == 0) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(to), "v"(off), "s"(rc) : "memory");
    else if (i % 4 == 1) asm volatile("buffer_load_dwordx4 %0, %1, 0 offen offset:%2 lds" :: "v"(off), "s"(rc), "n"(1 * 1024) : "memory");
    else if (i % 4 == 2) asm volatile("buffer_load_dwordx4 %0, %1, 0 offen offset:%2 lds" :: "v"(off), "s"(rc), "n"(2 * 1024) : "memory");
    else asm volatile("buffer_load_dwordx4 %0, %1, 0 offen offset:%2 lds" :: "v"(off), "s"(rc), "n"(3 * 1024) : "memory");
  };

  floatx4 acc[BW][BX];
#pragma unroll
  for (int i = 0; i < BW; ++i)
#pragma unroll
    for (int j = 0; j < BX; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int wrow = (wn * TN * 32 + r16) * 128, xrow = (BN + wm * TM * 32 + r16) * 128;
  // chunk c of the lane's row of block i of w or x, in one of the two stages
  auto read = [&](bool is_x, int stage, int i, int c) __attribute__((always_inline)) -> u32x4 {
    return *(const u32x4*)(Lds::at() + stage * STAGE + (is_x ? xrow : wrow) + i * 2048 + ((c ^ (r16 >> 1)) << 4));
  };

  // Loads of step t + 2 have places behind the products, from the barrier of step t on: place s of the 2 M up to the next barrier, the last quarter of which stays free for them to arrive.
  auto load_place = [&](int t, int stage, auto place) __attribute__((always_inline)) {
    constexpr int S = 3 * M / 2, first = (place() * L + S - 1) / S, last = ((place() + 1) * L + S - 1) / S;
    unrolled<(last < L ? last : L) - (first < L ? first : L)>([&](auto q) __attribute__((always_inline)) { issue(t, stage, first + q()); });
  };
  constexpr int FIRST = (M * L + 3 * M / 2 - 1) / (3 * M / 2);        // loads with places before M

  load_exps(0); place_exps(0);
  load_exps(1); place_exps(1);
#pragma unroll
  for (int t = 0; t < D; ++t) issue_exps(t);
#pragma unroll
  for (int t = 0; t < D - 1; ++t) {
    cut(t);
#pragma unroll
    for (int q = 0; q < L; ++q) issue(t, t, q);
  }
  cut(D - 1);
  unrolled<M>([&](auto p) __attribute__((always_inline)) { load_place(D - 1, D - 1, p); });
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"((D - 2) * L + FIRST) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  load_exps(2);

  // Loads and reads beyond the last step are of nothing (zeros go to LDS).  Reads and loads stand between the products, in the order of the code: a product keeps the matrix unit busy for 16 cycles or more, in which the wavefront issues what lies behind it.
  auto turn = [&](int t) __attribute__((always_inline)) {             // all are done with step t's place in LDS, and step t + 1 is there
    place_exps(t + 2);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"((D - 2) * L) : "memory");     // the loads of the D - 2 steps behind it may be under way
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    load_exps(t + 3);
    issue_exps(t + D);
    cut(t + D);
  };
  if constexpr (MX && !EXACT) {
    // A step is one product of k.  Its M products go through four quarters, (w low, x low), (w low, x high), (w high, x high), (w high, x low); each half of an operand is read
    // again, for the next use, as soon as the quarter that needed it last is over, so one set of registers does.  Odd steps have x low and high the other way round.
    u32x4 fw[BW][2], fx[BX][2];
    int ew[BW], ex[BX];
    auto fetch = [&](bool is_x, int stage, int high, int r) __attribute__((always_inline)) {      // read r of 3 TN or 3 TM of a half
      const int i = high * (is_x ? TM : TN) + r / 3, h = r % 3, at = is_x ? BN + wm * TM * 32 : wn * TN * 32;
      if (h == 2) {
        (is_x ? ex[is_x ? i : 0] : ew[is_x ? 0 : i]) = *(const uint8_t*)(Lds::at() + D * STAGE + (stage * EXPS + at + i * 16 + r16) * 4 + g);
      } else {
        (is_x ? fx[is_x ? i : 0][h & 1] : fw[is_x ? 0 : i][h & 1]) = read(is_x, stage, i, g + 4 * h);
      }
    };
#pragma unroll
    for (int r = 0; r < 3 * TN; ++r) fetch(false, 0, 0, r);
#pragma unroll
    for (int r = 0; r < 3 * TM; ++r) fetch(true, 0, 0, r);
    auto step = [&](int t, auto odd) __attribute__((always_inline)) {
      constexpr int X = odd() ? 1 : 0;                                // the half of x that comes first
      const int here = D == 2 ? X : t & (D - 1), next = D == 2 ? 1 - X : (t + 1) & (D - 1), before = D == 2 ? 1 - X : (t - 1) & (D - 1);      // places of this step, the next and the last
      unrolled<4>([&](auto quarter_) __attribute__((always_inline)) {
        constexpr int quarter = quarter_(), MQ = TN * TM, wh = quarter / 2, xh = (quarter == 1 || quarter == 2) ? 1 - X : X, R = quarter == 0 || quarter == 3 ? 3 * TM : 3 * TN;
        if constexpr (quarter == 2) turn(t);
        unrolled<MQ>([&](auto m_) __attribute__((always_inline)) {
          constexpr int m = m_(), i = wh * TN + m / TM, j = xh * TM + m % TM, first = (m * R + MQ - 1) / MQ, last = ((m + 1) * R + MQ - 1) / MQ;
          acc[i][j] = mfma_mx8(fw[i], fx[j], acc[i][j], ew[i], ex[j]);
          // quarter 0 reads the other half of x, 1 the other half of w, 2 the first half of w of the next step, 3 the half of x that the next step begins with
          unrolled<last - first>([&](auto d) __attribute__((always_inline)) {
            constexpr int r = first + d();
            if constexpr (quarter == 0) fetch(true, here, 1 - X, r);
            else if constexpr (quarter == 1) fetch(false, here, 1, r);
            else if constexpr (quarter == 2) fetch(false, next, 0, r);
            else fetch(true, next, 1 - X, r);
          });
          // the barrier lies between quarters 1 and 2
          constexpr int place = (quarter * MQ + m + 2 * MQ) % (4 * MQ) * 2;
          load_place(quarter >= 2 ? t + D : t + D - 1, quarter >= 2 ? here : before, std::integral_constant<int, place>{});
          load_place(quarter >= 2 ? t + D : t + D - 1, quarter >= 2 ? here : before, std::integral_constant<int, place + 1>{});
          __builtin_amdgcn_sched_barrier(0);
        });
      });
    };
#pragma nounroll
    for (int t = 0; t < nk; t += 2) { step(t, std::false_type{}); step(t + 1, std::true_type{}); }
  } else if constexpr (MX) {
    // A step is two halves of k.  An operand is widened shortly before its first product: a row of w during the row of products before its own, x along the first row.  What it was widened
    // from is read again at once, for the next half, so one set of registers does for what lies in LDS (256 x 256: 64 of it, 80 widened, 16 of exponents beside the sums' 256).
    u32x4 fw[BW], fx[BX], w16[2][2], x16[BX][2];
    unsigned ew[BW], ex[BX];
    auto fetch = [&](bool is_x, int t, int kq, int i) __attribute__((always_inline)) { (is_x ? fx[is_x ? i : 0] : fw[is_x ? 0 : i]) = read(is_x, t & (D - 1), i, 4 * kq + g); };
    auto scale = [&](bool is_x, int t, int i) __attribute__((always_inline)) {
      (is_x ? ex[is_x ? i : 0] : ew[is_x ? 0 : i]) =
          *(const unsigned*)(Lds::at() + D * STAGE + ((t & (RING - 1)) * EXPS + (is_x ? BN + wm * TM * 32 : wn * TN * 32) + i * 16 + r16) * 4);
    };
#pragma unroll
    for (int i = 0; i < BW; ++i) { fetch(false, 0, 0, i); scale(false, 0, i); }
#pragma unroll
    for (int j = 0; j < BX; ++j) { fetch(true, 0, 0, j); scale(true, 0, j); }
    auto step = [&](int t) __attribute__((always_inline)) {
      unrolled<2>([&](auto kq_) __attribute__((always_inline)) {
        constexpr int kq = kq_();
        if constexpr (kq == 1) turn(t);
        const int shift = 16 * kq + 8 * (g >> 1);
        // a quarter of 16 values of block i at a time, then the next half's in their place
        auto widen = [&](bool is_x, int i, int part) __attribute__((always_inline)) {
          const u32x4 v = is_x ? fx[is_x ? i : 0] : fw[is_x ? 0 : i];
          u32x4& to = is_x ? x16[is_x ? i : 0][part] : w16[i & 1][part];
          to = widen_mx8(v[2 * part], v[2 * part + 1], (is_x ? ex[is_x ? i : 0] : ew[is_x ? 0 : i]) >> shift & 255);
          if (part == 1) {
            fetch(is_x, t + kq, kq ^ 1, i);
            if (kq == 1) scale(is_x, t + 1, i);
          }
        };
        widen(false, 0, 0); widen(true, 0, 0); widen(false, 0, 1); widen(true, 0, 1);
        unrolled<M>([&](auto m_) __attribute__((always_inline)) {
          constexpr int m = m_(), i = m / BX, j = m % BX;
          unrolled<2>([&](auto part_) __attribute__((always_inline)) {
            constexpr int part = part_();
            acc[i][j] = mfma16<__bf16>(w16[i & 1][part], x16[j][part], acc[i][j]);
            if constexpr (i == 0 && j + 1 < BX) widen(true, j + 1, part);
            if constexpr (i + 1 < BW && j == BX - 2 + part) widen(false, i + 1, part);
            if constexpr (part == 1) load_place(kq == 1 ? t + D : t + D - 1, (kq == 1 ? t : t - 1) & (D - 1), std::integral_constant<int, kq == 1 ? m : M + m>{});
            __builtin_amdgcn_sched_barrier(0);
          });
        });
      });
    };
#pragma nounroll
    for (int t = 0; t < nk; ++t) step(t);
  } else {
    // A step is two products of k; two sets of operands.
    constexpr int R = BW + BX;
    u32x4 fw[2][BW], fx[2][BX];
    // read r of an operand set, in the order in which the products want them: the first row of w, all of x, the other rows of w
    auto fetch = [&](int set, int t, int kq, int r) __attribute__((always_inline)) {
      if (r >= 1 && r <= BX) fx[set][r - 1] = read(true, t & (D - 1), r - 1, 4 * kq + g);
      else fw[set][r ? r - BX : 0] = read(false, t & (D - 1), r ? r - BX : 0, 4 * kq + g);
    };
#pragma unroll
    for (int r = 0; r < R; ++r) fetch(0, 0, 0, r);
    auto step = [&](int t) __attribute__((always_inline)) {
      unrolled<2>([&](auto kq_) __attribute__((always_inline)) {
        constexpr int kq = kq_();
        if constexpr (kq == 1) turn(t);
        unrolled<M>([&](auto m_) __attribute__((always_inline)) {
          constexpr int m = m_(), i = m / BX, j = m % BX, first = (m * R + M - 1) / M, last = ((m + 1) * R + M - 1) / M;
          acc[i][j] = mfma_part<T>(fw[kq][i], fx[kq][j], acc[i][j]);
          unrolled<last - first>([&](auto d) __attribute__((always_inline)) { fetch(kq ^ 1, t + kq, kq ^ 1, first + d()); });
          load_place(kq == 1 ? t + D : t + D - 1, (kq == 1 ? t : t - 1) & (D - 1), std::integral_constant<int, kq == 1 ? m : M + m>{});
          __builtin_amdgcn_sched_barrier(0);
        });
      });
    };
#pragma nounroll
    for (int t = 0; t < nk; ++t) step(t);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

  if (a.direct) {
    const int col0 = n0 + (a.gated ? wn * TN * 16 : wn * TN * 32), tok0 = m0 + wm * TM * 32;
    if (a.y_kind == PRODUCT_Y_MX8) finish_direct<DirectMx8, TN, TM>(a, acc, n, tok0, col0, lane);
    else if (a.y_kind == PRODUCT_Y_F16) { if constexpr (!std::is_same<T, __bf16>::value && sizeof(T) < 4) finish_direct<_Float16, TN, TM>(a, acc, n, tok0, col0, lane); }
    else if constexpr (!std::is_same<T, _Float16>::value && sizeof(T) < 4) finish_direct<__bf16, TN, TM>(a, acc, n, tok0, col0, lane);
    return;
  }
  // Sums leave through LDS, up to 64 tokens of a wavefront at a time, in a place of its own: lanes then hold four neighbouring outputs of a token.  Chunks of four lie at their
  // number xor the token's.
  __syncthreads();
  float* const out = (float*)(Lds::at() + wave * UNIT);
  const int lpt_log2 = (TN == 4 ? 5 : 4) - a.gated, lpt = 1 << lpt_log2;      // lanes of a token
#pragma unroll
  for (int h = 0; h < TM; h += HT) {
#pragma unroll
    for (int j = 0; j < 2 * HT; ++j)
#pragma unroll
      for (int i = 0; i < BW; ++i) *(floatx4*)(out + ((j * 16 + r16) * TN * 8 + ((4 * i + g) ^ r16)) * 4) = acc[i][2 * h + j];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const int token0 = m0 + (wm * TM + h) * 32;
    auto piece = [&](int p, bool* on, int* i, int* j, floatx4* z, floatx4* up) __attribute__((always_inline)) {
      const int tok = p >> lpt_log2, o4 = p & (lpt - 1);
      const int c4 = a.gated ? o4 / 8 * 16 + o4 % 8 : o4;            // the chunk of its sums; those it is a gate of lie eight further on
      const float* const row = out + tok * TN * 32;
      *z = *(const floatx4*)(row + (c4 ^ (tok & 15)) * 4);
      *up = a.gated ? *(const floatx4*)(row + ((c4 + 8) ^ (tok & 15)) * 4) : *z;
      *i = token0 + tok; *j = n0 + wn * (lpt * 4) + o4 * 4; *on = *i < n && *j < a.cols;
    };
    constexpr int B = 4;
    static_assert(HT * 32 * TN * 4 % (64 * B) == 0, "whole batches");
    auto batches = [&](auto y) __attribute__((always_inline)) {
#pragma nounroll
      for (int p0 = lane; p0 < HT * 32 * lpt; p0 += 64 * B) {
        bool on[B]; int i[B], j[B]; floatx4 z[B], up[B];
#pragma unroll
        for (int b = 0; b < B; ++b) piece(p0 + 64 * b, &on[b], &i[b], &j[b], &z[b], &up[b]);
        product_finish_vec<decltype(y), B>(a, on, i, j, z, up);
      }
    };
    if (!a.vec) {
#pragma nounroll
      for (int p = lane; p < HT * 32 * lpt; p += 64) {
        bool on; int i, j; floatx4 z, up;
        piece(p, &on, &i, &j, &z, &up);
        product_finish4(a, i < n, i, j, z, up);
      }
    } else if (a.y_kind == PRODUCT_Y_F32) {
      batches(float{});
    } else if (a.y_kind == PRODUCT_Y_F16) {
      batches(_Float16{});
    } else {
      batches(__bf16{});
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
}

template <typename T, bool EXACT, int TN, int TM, int WN, int WM, int MINB, int D>
hipError_t launch_product_tile(ProductArgs a, hipStream_t s) {
  constexpr int BN = WN * TN * 32, BM = WM * TM * 32;
  const int outs = a.gated ? BN / 2 : BN;
  a.tiles_n = (a.cols + outs - 1) / outs; a.tiles_m = (a.n + BM - 1) / BM;
  const int lds = D == 2 ? 0 : ProductTile<T, EXACT, TN, TM, WN, WM, D>::LDS;
  if (lds) {
    static const bool ready = [lds] {     // more than 64 KB of dynamic LDS needs the attribute, once per instance
      (void)hipFuncSetAttribute((const void*)product_tile_kernel<T, EXACT, TN, TM, WN, WM, MINB, D>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
      (void)hipGetLastError();
      return true;
    }();
    (void)ready;
  }
  hipLaunchKernelGGL((product_tile_kernel<T, EXACT, TN, TM, WN, WM, MINB, D>), dim3((unsigned)(a.tiles_n * a.tiles_m)), dim3(WN * WM * 64), lds, s, a);
  return hipGetLastError();
}

// ---- few tokens: operands straight from memory ---------------------------------------------------------------------------
// The bound is memory: every weight goes into one or a few products.  A block makes TILES x 16 rows of w times TB x 16 tokens; its wavefronts take steps of 128 bytes of k in turn, load
// their operands from memory straight into registers, several steps in flight, and add up their sums in LDS at the end, in a fixed order.  A gated block has gates in the first
// half of its tiles and what they are a gate of in the second.  (64 tokens, 4096 -> 4096: bf16 17 us, fp32 34.)
template <typename T, int TILES, int TB>
__global__ __launch_bounds__(512, 2) void product_few_kernel(ProductArgs a) {
  constexpr bool MX = std::is_same<T, f8>::value;
  constexpr int W = 8, U = TILES + TB <= 3 ? 4 : 2;
  __shared__ __attribute__((aligned(16))) floatx4 red[W][TILES][TB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
  const int n = product_tokens(a);
  const int outs = a.gated ? TILES * 8 : TILES * 16;
  const int tn = blockIdx.x % a.tiles_n, tm = blockIdx.x / a.tiles_n;
  const int m0 = tm * TB * 16, n0 = tn * outs;
  if (m0 >= n) return;
  const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void*)(a.x + m0 * a.x_row), 0, 0x7FFFFFFF, BUF_FLAGS);
  const char* const w0 = a.w + n0 * a.w_row;
  const __amdgpu_buffer_rsrc_t rw[2] = {__builtin_amdgcn_make_buffer_rsrc((void*)w0, 0, 0x7FFFFFFF, BUF_FLAGS),
                                        __builtin_amdgcn_make_buffer_rsrc((void*)(w0 + (a.gated ? a.cols * a.w_row : 0)), 0, 0x7FFFFFFF, BUF_FLAGS)};
  __amdgpu_buffer_rsrc_t re[2], rxe;
  if constexpr (MX) {
    const uint8_t* const e0 = a.we + n0 * a.we_row;
    re[0] = __builtin_amdgcn_make_buffer_rsrc((void*)e0, 0, 0x7FFFFFFF, BUF_FLAGS);
    re[1] = __builtin_amdgcn_make_buffer_rsrc((void*)(e0 + (a.gated ? a.cols * a.we_row : 0)), 0, 0x7FFFFFFF, BUF_FLAGS);
    rxe = __builtin_amdgcn_make_buffer_rsrc((void*)(a.xe + m0 * a.xe_row), 0, 0x7FFFFFFF, BUF_FLAGS);
  }
  int woff[TILES], weoff[TILES], xoff[TB], xeoff[TB];
#pragma unroll
  for (int i = 0; i < TILES; ++i) {
    const int col = (a.gated ? i % (TILES > 1 ? TILES / 2 : 1) : i) * 16 + r16;
    woff[i] = n0 + col < a.cols ? col * (int)a.w_row + g * 16 : OOB;
    weoff[i] = n0 + col < a.cols ? col * (int)a.we_row + g / 2 : OOB;
  }
#pragma unroll
  for (int j = 0; j < TB; ++j) {
    const bool there = m0 + j * 16 + r16 < n;
    xoff[j] = there ? (j * 16 + r16) * (int)a.x_row + g * 16 : OOB;
    xeoff[j] = there ? (j * 16 + r16) * (int)a.xe_row + g / 2 : OOB;
  }
  const int nk = (a.k_bytes + 127) / 128;
  floatx4 acc[TILES][TB];
#pragma unroll
  for (int i = 0; i < TILES; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

  for (int t0 = wave; t0 < nk; t0 += W * U) {
    u32x4 fw[U][TILES][2], fx[U][TB][2];
    unsigned ew[U][TILES][2], ex[U][TB][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * W;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        // chunks g and g + 4 of the step; beyond the row's end, and for steps beyond the last, zeros that no memory is asked for
        const int beyond = t * 128 + h * 64 + g * 16 >= a.k_bytes ? OOB : 0;
#pragma unroll
        for (int i = 0; i < TILES; ++i)
          fw[u][i][h] = __builtin_amdgcn_raw_buffer_load_b128(rw[a.gated && i >= TILES / 2], (woff[i] | beyond) + t * 128 + h * 64, 0, 0);
#pragma unroll
        for (int j = 0; j < TB; ++j) fx[u][j][h] = __builtin_amdgcn_raw_buffer_load_b128(rx, (xoff[j] | beyond) + t * 128 + h * 64, 0, 0);
        if constexpr (MX) {
#pragma unroll
          for (int i = 0; i < TILES; ++i) ew[u][i][h] = __builtin_amdgcn_raw_buffer_load_b8(re[a.gated && i >= TILES / 2], (weoff[i] | beyond) + t * 4 + h * 2, 0, 0);
#pragma unroll
          for (int j = 0; j < TB; ++j) ex[u][j][h] = __builtin_amdgcn_raw_buffer_load_b8(rxe, (xeoff[j] | beyond) + t * 4 + h * 2, 0, 0);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (MX) {
          u32x4 w[TILES][2], x[TB][2];
#pragma unroll
          for (int i = 0; i < TILES; ++i) widen_mx8(fw[u][i][h], ew[u][i][h], &w[i][0], &w[i][1]);
#pragma unroll
          for (int j = 0; j < TB; ++j) widen_mx8(fx[u][j][h], ex[u][j][h], &x[j][0], &x[j][1]);
#pragma unroll
          for (int i = 0; i < TILES; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j) acc[i][j] = mfma16<__bf16>(w[i][1], x[j][1], mfma16<__bf16>(w[i][0], x[j][0], acc[i][j]));
        } else if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int i = 0; i < TILES; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j) {
              const floatx4 w = __builtin_bit_cast(floatx4, fw[u][i][h]), x = __builtin_bit_cast(floatx4, fx[u][j][h]);
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], x[e], acc[i][j], 0, 0, 0);
            }
        } else {
#pragma unroll
          for (int i = 0; i < TILES; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j) acc[i][j] = mfma16<T>(fw[u][i][h], fx[u][j][h], acc[i][j]);
        }
      }
  }
#pragma unroll
  for (int i = 0; i < TILES; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) red[wave][i][j][lane] = acc[i][j];
  __syncthreads();
  // token l % 16 and rows 4 (l / 16) .. + 3 of a tile are lane l's
  const int quads = outs / 4;
  for (int p = threadIdx.x; p < quads * TB * 16; p += 512) {
    const int tok = p / quads, q = p % quads, at = (q & 3) * 16 + (tok & 15);
    floatx4 z = red[0][q >> 2][tok >> 4][at], up = z;
    for (int w = 1; w < W; ++w) z += red[w][q >> 2][tok >> 4][at];
    if (a.gated) {
      const int second = (q >> 2) + TILES / 2;
      up = red[0][second % TILES][tok >> 4][at];
      for (int w = 1; w < W; ++w) up += red[w][second % TILES][tok >> 4][at];
    }
    product_finish4(a, m0 + tok < n, m0 + tok, n0 + q * 4, z, up);
  }
}

template <typename T, int TILES, int TB>
hipError_t launch_product_few(ProductArgs a, hipStream_t s) {
  const int outs = a.gated ? TILES * 8 : TILES * 16;
  a.tiles_n = (a.cols + outs - 1) / outs; a.tiles_m = (a.n + TB * 16 - 1) / (TB * 16);
  hipLaunchKernelGGL((product_few_kernel<T, TILES, TB>), dim3((unsigned)(a.tiles_n * a.tiles_m)), dim3(512), 0, s, a);
  return hipGetLastError();
}

// ---- up to 16 tokens: x stays in registers -----------------------------------------------------------------------------------
// As above, but a block takes one group of TILES x 16 rows of w after the other, and its wavefronts keep their parts of x, XS steps, for all of them: x is read once a block and not once a
// group (16 tokens, 4096 -> 131072 bf16: 253 us of reading x with every group).  The weights of the next steps, also of the next group's first, are on their way while products
// and sums of the present ones are made.  Rows of 8 bits have their exponents in aligned words.
template <typename T, int TILES, int XS>
__global__ __launch_bounds__(512, 2) void product_held_kernel(ProductArgs a) {
  constexpr bool MX = std::is_same<T, f8>::value;
  constexpr int W = 8, U = XS > 4 && TILES == 1 && !(MX && XS > 8) ? 4 : 2, C = XS / U;  // steps of a part, parts of a group: an even number
  __shared__ __attribute__((aligned(16))) floatx4 red[2][W][TILES][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
  const int n = product_tokens(a);
  if (n == 0) return;
  const int outs = a.gated ? TILES * 8 : TILES * 16, nk = (a.k_bytes + 127) / 128;
  // chunks g and g + 4 of a step; beyond a row's end, and for steps beyond the last, zeros that no memory is asked for
  auto beyond = [&](int t, int h) __attribute__((always_inline)) { return t * 128 + h * 64 + g * 16 >= a.k_bytes ? OOB : 0; };

  u32x4 fx[XS][2];
  unsigned ex[MX ? XS : 1];
  {
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void*)a.x, 0, 0x7FFFFFFF, BUF_FLAGS), rxe = __builtin_amdgcn_make_buffer_rsrc((void*)a.xe, 0, 0x7FFFFFFF, BUF_FLAGS);
    const int xoff = r16 < n ? r16 * (int)a.x_row + g * 16 : OOB, xeoff = r16 < n ? r16 * (int)a.xe_row : OOB;
#pragma unroll
    for (int u = 0; u < XS; ++u) {
      const int t = wave + u * W;
#pragma unroll
      for (int h = 0; h < 2; ++h) fx[u][h] = __builtin_amdgcn_raw_buffer_load_b128(rx, (xoff | beyond(t, h)) + t * 128 + h * 64, 0, 0);
      if constexpr (MX) ex[u] = __builtin_amdgcn_raw_buffer_load_b32(rxe, (t < nk ? xeoff : OOB) + t * 4, 0, 0);
    }
  }
  u32x4 fw[2][U][TILES][2];
  unsigned ew[2][U][MX ? TILES : 1];
  auto load = [&](int buf, int group, int part) __attribute__((always_inline)) {
    const int n0 = group * outs;
    const char* const w0 = a.w + n0 * a.w_row;
    const __amdgpu_buffer_rsrc_t rw[2] = {__builtin_amdgcn_make_buffer_rsrc((void*)w0, 0, 0x7FFFFFFF, BUF_FLAGS),
                                          __builtin_amdgcn_make_buffer_rsrc((void*)(w0 + (a.gated ? a.cols * a.w_row : 0)), 0, 0x7FFFFFFF, BUF_FLAGS)};
    const uint8_t* const e0 = a.we + n0 * a.we_row;
    const __amdgpu_buffer_rsrc_t re[2] = {__builtin_amdgcn_make_buffer_rsrc((void*)e0, 0, 0x7FFFFFFF, BUF_FLAGS),
                                          __builtin_amdgcn_make_buffer_rsrc((void*)(e0 + (a.gated ? a.cols * a.we_row : 0)), 0, 0x7FFFFFFF, BUF_FLAGS)};
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const int col = (a.gated ? i % (TILES > 1 ? TILES / 2 : 1) : i) * 16 + r16;
      const bool second = a.gated && i >= TILES / 2, there = group < a.tiles_n && n0 + col < a.cols;
      const int woff = there ? col * (int)a.w_row + g * 16 : OOB, weoff = there ? col * (int)a.we_row : OOB;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = wave + (part * U + u) * W;
#pragma unroll
        for (int h = 0; h < 2; ++h) fw[buf][u][i][h] = __builtin_amdgcn_raw_buffer_load_b128(rw[second], (woff | beyond(t, h)) + t * 128 + h * 64, 0, 0);
        if constexpr (MX) ew[buf][u][i] = __builtin_amdgcn_raw_buffer_load_b32(re[second], (t < nk ? weoff : OOB) + t * 4, 0, 0);
      }
    }
  };
  load(0, blockIdx.x, 0);
  int turn = 0;
#pragma nounroll
  for (int group = blockIdx.x; group < a.tiles_n; group += gridDim.x, turn ^= 1) {
    floatx4 acc[TILES];
#pragma unroll
    for (int i = 0; i < TILES; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    if constexpr (MX)
#pragma unroll
      for (int u = 0; u < XS; ++u) asm volatile("" : "+v"(ex[u]));     // or every exponent's scale takes a register for the whole loop
#pragma unroll
    for (int part = 0; part < C; ++part) {
      if (part + 1 < C) load((part + 1) & 1, group, part + 1);
      else load(0, group + gridDim.x, 0);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int s = part * U + u, shift = 8 * (g >> 1) + 16 * h;
          u32x4 x[2];
          if constexpr (MX) widen_mx8(fx[s][h], ex[s] >> shift & 255, &x[0], &x[1]);
#pragma unroll
          for (int i = 0; i < TILES; ++i) {
            if constexpr (MX) {
              u32x4 w[2];
              widen_mx8(fw[part & 1][u][i][h], ew[part & 1][u][i] >> shift & 255, &w[0], &w[1]);
              acc[i] = mfma16<__bf16>(w[1], x[1], mfma16<__bf16>(w[0], x[0], acc[i]));
            } else {
              acc[i] = mfma_part<T>(fw[part & 1][u][i][h], fx[s][h], acc[i]);
            }
          }
        }
    }
#pragma unroll
    for (int i = 0; i < TILES; ++i) red[turn][wave][i][lane] = acc[i];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                // and not for the loads
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int quads = outs / 4;
    for (int p = threadIdx.x; p < quads * 16; p += 512) {
      const int tok = p / quads, q = p % quads, at = (q & 3) * 16 + tok;
      floatx4 z = red[turn][0][q >> 2][at], up = z;
      for (int w = 1; w < W; ++w) z += red[turn][w][q >> 2][at];
      if (a.gated) {
        const int second = ((q >> 2) + TILES / 2) % TILES;
        up = red[turn][0][second][at];
        for (int w = 1; w < W; ++w) up += red[turn][w][second][at];
      }
      product_finish4(a, tok < n, tok, group * outs + q * 4, z, up);
    }
  }
}

template <typename T, int TILES, int XS>
hipError_t launch_product_held(ProductArgs a, hipStream_t s) {
  constexpr int BLOCKS = 256;                                         // one a CU, whose wavefronts fill its registers
  const int outs = a.gated ? TILES * 8 : TILES * 16;
  a.tiles_n = (a.cols + outs - 1) / outs; a.tiles_m = 1;
  hipLaunchKernelGGL((product_held_kernel<T, TILES, XS>), dim3((unsigned)(a.tiles_n < BLOCKS ? a.tiles_n : BLOCKS)), dim3(512), 0, s, a);
  return hipGetLastError();
}
template <typename T, int TILES>
hipError_t launch_product_held_steps(const ProductArgs& a, hipStream_t s) {
  constexpr int MOST = product_held_steps(TILES, std::is_same<T, f8>::value);
  const int steps = (a.k_bytes + 1023) / 1024;
  if (steps <= 4) return launch_product_held<T, TILES, 4>(a, s);
  if constexpr (MOST >= 16) { if (steps > 8) return launch_product_held<T, TILES, 16>(a, s); }
  if constexpr (MOST >= 8) return launch_product_held<T, TILES, 8>(a, s);
  return hipErrorInvalidValue;
}

template <typename T> hipError_t launch_product(int variant, const ProductArgs& a, hipStream_t s);

#ifdef OCTO_PRODUCT_TYPE
template <> hipError_t launch_product<OCTO_PRODUCT_TYPE>(int variant, const ProductArgs& a, hipStream_t s) {
  typedef OCTO_PRODUCT_TYPE T;
  if constexpr (std::is_same<T, f8>::value) {
    if (a.exact8) {
      switch (variant) {
        case 1: return launch_product_tile<T, true, 4, 4, 2, 2, 1, 2>(a, s);
        case 2: return launch_product_tile<T, true, 2, 2, 2, 2, 2, 2>(a, s);
        case 3: return launch_product_tile<T, true, 2, 1, 2, 2, 2, 4>(a, s);
        case 4: return launch_product_tile<T, true, 2, 2, 2, 2, 2, 4>(a, s);
      }
    }
  } else {
    switch (variant) {
      case 22: return launch_product_few<T, 2, 2>(a, s);
      case 24: if constexpr (sizeof(T) == 2) return launch_product_few<T, 2, 4>(a, s); else break;
      case 42: if constexpr (sizeof(T) == 4) return launch_product_few<T, 4, 2>(a, s); else break;
      case 44: if constexpr (sizeof(T) == 4) return launch_product_few<T, 4, 4>(a, s); else break;
    }
  }
  switch (variant) {
    case 1: if constexpr (sizeof(T) < 4) return launch_product_tile<T, false, 4, 4, 2, 2, 1, 2>(a, s); else break;
    case 2: return launch_product_tile<T, false, 2, 2, 2, 2, 2, 2>(a, s);
    case 3: return launch_product_tile<T, false, 2, 1, 2, 2, 2, 4>(a, s);
    case 4: return launch_product_tile<T, false, 2, 2, 2, 2, 2, 4>(a, s);
    case 10: return launch_product_held_steps<T, 1>(a, s);
    case 20: return launch_product_held_steps<T, 2>(a, s);
    case 40: return launch_product_held_steps<T, 4>(a, s);
    case 11: return launch_product_few<T, 1, 1>(a, s);
    case 21: return launch_product_few<T, 2, 1>(a, s);
    case 41: return launch_product_few<T, 4, 1>(a, s);
  }
  return hipErrorInvalidValue;
}
#endif

}  // namespace octo
