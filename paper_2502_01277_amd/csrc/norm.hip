// octo_op_norm: residual sum and root-mean-square norm of rows, in their type or in 8 bits; octo_op_mx8_load and the host's conversions.
//
//   s = x + r,   y = s w / sqrt(mean s^2 + eps)
// The bound is memory: every value is read and written once against some ten operations.  8 bits are a coarse grid, and a value that fp32 puts on the other side of a border between two codes is
// off by a code (one in two million): sums are in fp64, and values near a border are looked at again in fp64 (all of them in fp64: 12800 x 4096 with residual 123 -> 167 us).  A row is held by `lanes` threads, `items` vectors of 16 bytes in each, as fp32
// from the load to the store: the sum of squares needs no second look at memory.  A group of 32 that goes to 8 bits lies in four (fp32: eight) lanes
// beside each other, its largest magnitude comes from exchanges between them.
// Measured (MI355X): 12800 x 4096 bf16 with residual and sum to 8 bits 72 us, 5.1 TB/s, and back to bf16 27; 14700 x 256 fp32 with residual and sum 10.
#include <cmath>
#include <cstring>

#include "mx8.h"
#include "octo_internal.h"

namespace octo {
namespace {

struct NormArgs {
  const void* x; const void* res; void* sum; void* y;
  long long x_row, res_row, sum_row, y_row;
  octo_mx8_rows y8;
  const float* w;
  const int* n_dyn;
  int n, width, norm, w_aligned;
  float eps;
};

template <typename T, int VEC> struct alignas(sizeof(T) * VEC) NormPack { T v[VEC]; };

// To fp32 on the way to 8 bits: the last bit is set where something was cut off, so that the second rounding gives what one would.
__device__ __forceinline__ float narrow(double v) {
  const float f = (float)v;
  const double back = (double)f;
  const unsigned bits = __float_as_uint(f);
  // the neighbour of odd bits on the side of v: f itself if it is odd
  const unsigned toward = fabs(back) < fabs(v) ? bits + 1u : bits - 1u;
  return back == v || (bits & 1u) || !(fabs(v) < 3.4e38) ? f : __uint_as_float(toward);
}

// A block of 256 threads holds 256 / LANES rows, or one of 1024 one row.  Element (i, t, e) of a row is (i LANES + t) VEC + e.
template <typename T, int VEC, int LANES, int ITEMS, bool TO8>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void norm_kernel(NormArgs a) {
  constexpr int THREADS_ = LANES > 256 ? LANES : 256, ROWS = THREADS_ / LANES, WAVES = (LANES + 63) / 64;
  typedef NormPack<T, VEC> P;
  const int at = threadIdx.x % LANES, row = blockIdx.x * ROWS + threadIdx.x / LANES;
  const int n = a.n_dyn ? min(max(*a.n_dyn, 0), a.n) : a.n;
  if (WAVES == 1 && row >= n) return;                   // lanes of a row come and go together
  const bool there = row < n;                           // rows of several wavefronts meet at a barrier
  P in[ITEMS], more[ITEMS];
  const T* x = (const T*)a.x + row * a.x_row;
  const T* r = (const T*)a.res + row * a.res_row;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int c = (i * LANES + at) * VEC;
    if (there && c < a.width) in[i] = *(const P*)(x + c);
  }
  if (a.res) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = (i * LANES + at) * VEC;
      if (there && c < a.width) more[i] = *(const P*)(r + c);
    }
  }
  float u[ITEMS][VEC];
  double total = 0.0;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const bool any = there && (i * LANES + at) * VEC < a.width;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      u[i][e] = any ? (float)in[i].v[e] : 0.f;
      if (a.res && any) u[i][e] += (float)more[i].v[e];
      total = fma((double)u[i][e], (double)u[i][e], total);
    }
  }
  double f = 1.0;
  if (a.norm) {
#pragma unroll
    for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) total += __shfl_xor(total, d);
    if constexpr (WAVES > 1) {
      __shared__ double part[THREADS_ / 64];
      if (!(threadIdx.x & 63)) part[threadIdx.x >> 6] = total;
      __syncthreads();
      const int first = threadIdx.x / LANES * WAVES;
      total = 0.0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) total += part[first + w];
    }
    f = 1.0 / sqrt(total / a.width + (double)a.eps);
  }
  const float f32 = (float)f;
  if (WAVES > 1 && !there) return;
  if (a.sum) {
    T* s = (T*)a.sum + row * a.sum_row;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = (i * LANES + at) * VEC;
      if (c >= a.width) continue;
      P o;
#pragma unroll
      for (int e = 0; e < VEC; ++e) o.v[e] = (T)u[i][e];
      *(P*)(s + c) = o;
    }
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int c = (i * LANES + at) * VEC;
    if (c >= a.width) continue;                         // the lanes of a group come and go together too
#pragma unroll
    for (int e = 0; e < VEC; ++e) asm volatile("" : "+v"(u[i][e]));         // fp64 copies of the sum are not kept until here
    float w[VEC], y[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[e] = 1.0f;
    if (a.w) {
      if (VEC % 4 == 0 && a.w_aligned) {
#pragma unroll
        for (int e = 0; e < VEC; e += 4) {
          const floatx4 v = *(const floatx4*)(a.w + c + e);
#pragma unroll
          for (int k = 0; k < 4; ++k) w[e + k] = v[k];
        }
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[e] = a.w[c + e];
      }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) y[e] = !TO8 && sizeof(T) == 4 ? (float)((double)u[i][e] * f * (double)w[e]) : u[i][e] * f32 * w[e];
    if constexpr (TO8) {
      auto largest = [&]() __attribute__((always_inline)) {
        unsigned most = 0;                              // magnitudes compare as integers
#pragma unroll
        for (int e = 0; e < VEC; ++e) most = max(most, __float_as_uint(y[e]) & 0x7FFFFFFFu);
#pragma unroll
        for (int d = 1; d < 32 / VEC; d *= 2) most = max(most, (unsigned)__shfl_xor((int)most, d));
        return most;
      };
      unsigned most = largest();
      float inverse = mx8_inverse(mx8_exp(most));
      // fp32 is off by up to four last bits.  Is a value that near to the middle between two codes (of 3 bits behind the point), or among the codes without a leading one, or the
      // largest that near to where the exponent changes?  Then the wavefront takes all of them in fp64.
      bool near = (most + 8u - 0x600000u & 0x7FFFFFu) < 16u;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const unsigned bits = __float_as_uint(y[e] * inverse) & 0x7FFFFFFFu;
        near = near || (bits + 8u - 0x80000u & 0xFFFFFu) < 16u || bits - 1u < 0x3C800000u - 1u;
      }
      if ((a.norm || a.w) && __any(near)) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) y[e] = narrow((double)u[i][e] * f * (double)w[e]);
        most = largest();
        inverse = mx8_inverse(mx8_exp(most));
      }
      const bool none = most >= 0x7F800000u;
      uint8_t* q = a.y8.d_codes + row * a.y8.code_row + c;
      unsigned o[VEC / 4];
#pragma unroll
      for (int e = 0; e < VEC; e += 4) o[e / 4] = none ? MX8_NAN4 : mx8_pack4(floatx4{y[e], y[e + 1], y[e + 2], y[e + 3]}, inverse);
      if constexpr (VEC == 8) *(u32x2*)q = u32x2{o[0], o[1]};
      else *(unsigned*)q = o[0];
      if (c % 32 == 0) a.y8.d_exps[row * a.y8.exp_row + c / 32] = (uint8_t)(none ? 255 : mx8_exp(most));
    } else {
      P o;
#pragma unroll
      for (int e = 0; e < VEC; ++e) o.v[e] = (T)y[e];
      *(P*)((T*)a.y + row * a.y_row + c) = o;
    }
  }
}

template <typename T, int VEC, int LANES, int ITEMS, bool TO8>
hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  constexpr int threads = LANES > 256 ? LANES : 256, rows = threads / LANES;
  if ((unsigned long long)a.n * LANES > 0xFFFF0000ull) return hipErrorInvalidValue;      // HIP counts the threads of a launch in 32 bits
  hipLaunchKernelGGL((norm_kernel<T, VEC, LANES, ITEMS, TO8>), dim3((unsigned)((a.n + rows - 1) / rows)), dim3(threads), 0, s, a);
  return hipGetLastError();
}

// Threads of a row: as few as hold it in 32 values each (64 values of 16 bits take 170 registers: 12800 x 4096 bf16 with residual to 8 bits 137 us, 32 values 76), more where that would
// leave the chip without wavefronts.
template <typename T, int VEC, bool TO8>
hipError_t launch_norm_vec(const NormArgs& a, hipStream_t s) {
  constexpr int MOST = 32 / VEC < 8 ? 32 / VEC : 8;
  const int vectors = (a.width + VEC - 1) / VEC;
  auto items_of = [&](int lanes) { int i = 1; while (lanes * i < vectors) i *= 2; return i; };
  int lanes = 16;
  while (lanes < 1024 && (items_of(lanes) > MOST || (items_of(lanes) > 1 && (long long)a.n * lanes < 65536))) lanes *= 4;
  const int items = items_of(lanes);
#define OCTO_NORM(L, I) if (lanes == L && items == I) return launch_norm<T, VEC, L, I, TO8>(a, s);
#define OCTO_NORM_ITEMS(L) OCTO_NORM(L, 1) OCTO_NORM(L, 2) OCTO_NORM(L, 4) if constexpr (MOST == 8) { OCTO_NORM(L, 8) }
  OCTO_NORM_ITEMS(16) OCTO_NORM_ITEMS(64) OCTO_NORM_ITEMS(256) OCTO_NORM_ITEMS(1024)
  if constexpr (VEC == 1) { OCTO_NORM(1024, 16) OCTO_NORM(1024, 32) }
#undef OCTO_NORM_ITEMS
#undef OCTO_NORM
  return hipErrorInvalidValue;
}

template <typename T>
hipError_t launch_norm_type(const NormArgs& a, bool to8, int vec, hipStream_t s) {
  constexpr int N = 16 / sizeof(T);
  if (to8) return launch_norm_vec<T, N, true>(a, s);
  if (vec == N) return launch_norm_vec<T, N, false>(a, s);
  return launch_norm_vec<T, 1, false>(a, s);
}

struct Mx8Args {
  octo_mx8_rows x; void* y; long long y_row;
  const int* n_dyn; int n; unsigned chunks, total; FastDiv div_chunks;
};

// A thread makes 16 bytes of values.
template <typename T>
__global__ __launch_bounds__(256) void mx8_load_kernel(Mx8Args a) {
  constexpr int CH = 16 / sizeof(T);
  const unsigned i = blockIdx.x * 256u + threadIdx.x;
  if (i >= a.total) return;
  const unsigned row = fast_div(i, a.div_chunks), c = (i - row * a.chunks) * CH;
  if (a.n_dyn && (int)row >= *a.n_dyn) return;
  const uint8_t* const codes = a.x.d_codes + row * a.x.code_row + c;
  const int ex = a.x.d_exps[row * a.x.exp_row + c / 32];
  const float scale = mx8_scale(ex);
  auto widen = [&](unsigned w) {
    floatx4 v = f8_unpack4(w);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = ex == 255 ? __builtin_nanf("") : v[e] * scale;
    return v;
  };
  T* y = (T*)a.y + row * a.y_row + c;
  if constexpr (sizeof(T) == 4) {
    __builtin_nontemporal_store(widen(*(const unsigned*)codes), (floatx4*)y);
  } else {
    const u32x2 w = *(const u32x2*)codes;
    u32x4 o;
    store4<T>((T*)&o, widen(w[0]));
    store4<T>((T*)&o + 4, widen(w[1]));
    __builtin_nontemporal_store(o, (u32x4*)y);
  }
}

bool token_dtype(int dt) { return dt == OCTO_F32 || dt == OCTO_F16 || dt == OCTO_BF16; }

}  // namespace
}  // namespace octo

using namespace octo;

extern "C" {

octo_status octo_op_norm(const octo_norm_op* op, void* hip_stream) {
  if (!op || !token_dtype(op->dtype) || (op->y_format != OCTO_ROWS_PLAIN && op->y_format != OCTO_ROWS_MX8)) return OCTO_EINVAL;
  if (op->n < 0 || op->width < 1 || op->width > 32768 || !op->d_x || (op->norm && !(op->eps >= 0))) return OCTO_EINVAL;
  if (op->x_row < 0 || (op->d_res && op->res_row < 0) || (op->d_sum && op->sum_row < 0)) return OCTO_EINVAL;
  if (op->d_sum && op->d_sum == op->d_y && op->y_format == OCTO_ROWS_PLAIN) return OCTO_EINVAL;
  const int es = op->dtype == OCTO_F32 ? 4 : 2;
  const bool to8 = op->y_format == OCTO_ROWS_MX8;
  if (to8 ? op->width % 32 || !mx8_ok(op->y8) : !op->d_y || op->y_row < 0) return OCTO_EINVAL;
  const uintptr_t at = (uintptr_t)op->d_x | (uintptr_t)op->d_res | (uintptr_t)op->d_sum | (to8 ? 0 : (uintptr_t)op->d_y);
  const long long rows = op->x_row | (op->d_res ? op->res_row : 0) | (op->d_sum ? op->sum_row : 0) | (to8 ? 0 : op->y_row);
  if (at % es || ((uintptr_t)op->d_weight & 3) || ((uintptr_t)op->d_n & 3)) return OCTO_EINVAL;
  const bool wide = !(at & 15) && !(rows * es & 15) && op->width % (16 / es) == 0;
  if (to8 && !wide) return OCTO_EINVAL;
  NormArgs a{};
  a.x = op->d_x; a.res = op->d_res; a.sum = op->d_sum; a.y = op->d_y;
  a.x_row = op->x_row; a.res_row = op->res_row; a.sum_row = op->sum_row; a.y_row = op->y_row;
  a.y8 = op->y8; a.w = op->d_weight; a.n_dyn = op->d_n; a.n = op->n; a.width = op->width; a.norm = op->norm;
  a.w_aligned = !((uintptr_t)op->d_weight & 15);
  a.eps = op->eps;
  if (!op->n) return OCTO_OK;
  hipStream_t s = (hipStream_t)hip_stream;
  const int vec = wide ? 16 / es : 1;
  const hipError_t e = op->dtype == OCTO_F32 ? launch_norm_type<float>(a, to8, vec, s) : op->dtype == OCTO_F16 ? launch_norm_type<_Float16>(a, to8, vec, s) : launch_norm_type<__bf16>(a, to8, vec, s);
  return e == hipSuccess ? OCTO_OK : e == hipErrorInvalidValue ? OCTO_EINVAL : OCTO_EHIP;
}

octo_status octo_op_mx8_load(const octo_mx8_op* op, void* hip_stream) {
  if (!op || !token_dtype(op->dtype) || op->n < 0 || op->width < 32 || op->width % 32 || !mx8_ok(op->x8) || !op->d_y || op->y_row < 0) return OCTO_EINVAL;
  const int es = op->dtype == OCTO_F32 ? 4 : 2;
  if (((uintptr_t)op->d_y & 15) || (op->y_row * es & 15) || ((uintptr_t)op->d_n & 3)) return OCTO_EINVAL;
  const int ch = 16 / es;                                           // values a thread
  const long long total = (long long)op->n * (op->width / ch);
  if (total > 0x7FFFFF00ll) return OCTO_EINVAL;
  if (!total) return OCTO_OK;
  Mx8Args a{};
  a.x = op->x8; a.y = op->d_y; a.y_row = op->y_row; a.n_dyn = op->d_n; a.n = op->n;
  a.chunks = (unsigned)(op->width / ch); a.total = (unsigned)total; a.div_chunks = make_fastdiv(a.chunks);
  const dim3 grid((a.total + 255) / 256);
  hipStream_t s = (hipStream_t)hip_stream;
  if (op->dtype == OCTO_F32) hipLaunchKernelGGL(mx8_load_kernel<float>, grid, dim3(256), 0, s, a);
  else if (op->dtype == OCTO_F16) hipLaunchKernelGGL(mx8_load_kernel<_Float16>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(mx8_load_kernel<__bf16>, grid, dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? OCTO_OK : OCTO_EHIP;
}

octo_status octo_quantize_mx8(const float* src, size_t n, uint8_t* codes, uint8_t* exps) {
  if (n % 32 || ((!src || !codes || !exps) && n)) return OCTO_EINVAL;
  for (size_t g = 0; g < n / 32; ++g) {
    const float* x = src + 32 * g;
    float most = 0.f;
    bool finite = true;
    for (int i = 0; i < 32; ++i) { finite = finite && std::isfinite(x[i]); most = std::fmax(most, std::fabs(x[i])); }
    int e = -126;                                // the smallest exponent with most <= 448 * 2^e
    if (finite && most > 0.f) {
      int ex = 0;
      const float m = std::frexp(most, &ex);     // most = m * 2^ex, 0.5 <= m < 1
      e = m <= 0.875f ? ex - 9 : ex - 8;
      e = e < -126 ? -126 : e;
    }
    exps[g] = finite ? (uint8_t)(e + 127) : 255;
    if (!finite) { memset(codes + 32 * g, 0x7F, 32); continue; }
    float scaled[32];
    for (int i = 0; i < 32; ++i) scaled[i] = std::ldexp(x[i], -e);      // exact: what becomes subnormal in fp32 is far below a code's step
    const octo_status st = octo_quantize_e4m3(scaled, 32, 1.0f, codes + 32 * g);
    if (st != OCTO_OK) return st;
  }
  return OCTO_OK;
}

octo_status octo_dequantize_mx8(const uint8_t* codes, const uint8_t* exps, size_t n, float* dst) {
  if (n % 32 || ((!codes || !exps || !dst) && n)) return OCTO_EINVAL;
  const octo_status st = octo_dequantize_e4m3(codes, n, 1.0f, dst);
  if (st != OCTO_OK) return st;
  for (size_t i = 0; i < n; ++i) dst[i] = exps[i / 32] == 255 ? std::nanf("") : std::ldexp(dst[i], exps[i / 32] - 127);
  return OCTO_OK;
}

}  // extern "C"
