// The cache of 4 bits a value: octo_op_cache4_store / _load on the device, the same conversion on the host.
//
// The bound is memory.  A lane takes eight values of a group of 32, four lanes the group: the largest magnitude comes from two
// exchanges between neighbours, the exponent from its bits, the codes from the conversion instructions (E2M1 with a power-of-two scale, round to
// nearest even, saturating).  Loads and stores are 16 and 4 bytes a lane, in the order of the states.  What is read back from the cache goes past the
// caches' reuse order (51200 tokens: 83 -> 57 us), what is stored does not (its lines are filled by several wavefronts).
#include <cmath>
#include <cstring>

#include "mfma_common.h"
#include "octo_internal.h"

namespace octo {
namespace {

struct Cache4Args {
  octo_cache4_plane plane[2];
  void* x[2]; long long token[2], head[2];
  const long long* slots; const int* n_dyn;
  long long rows;
  int n, heads;
  FastDiv div_chunks, div_heads;     // chunks of eight values per head; heads
  unsigned chunks, total;            // chunks per head; per tensor
};

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <typename T> __device__ __forceinline__ void read8(const T* p, float* v) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const floatx4 f = load4(p + 4 * h);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * h + e] = f[e];
  }
}

// thread -> (tensor, token, head, chunk); false where there is none
__device__ __forceinline__ bool chunk_of(const Cache4Args& a, int* k, int* tok, int* head, int* chunk) {
  unsigned i = blockIdx.x * 256u + threadIdx.x;
  *k = blockIdx.y;
  if (i >= a.total) return false;
  const unsigned row = fast_div(i, a.div_chunks), t = fast_div(row, a.div_heads);
  *chunk = (int)(i - row * a.chunks); *tok = (int)t; *head = (int)(row - t * (unsigned)a.heads);
  return !a.n_dyn || *tok < *a.n_dyn;
}

template <typename T>
__device__ __forceinline__ void store_group(const octo_cache4_plane& p, const float* v, long long slot, int head, int chunk) {
  unsigned most = 0;                              // magnitudes compare as integers, infinities and NaN above all others
#pragma unroll
  for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(v[e]) & 0x7FFFFFFFu);
  most = max(most, (unsigned)__shfl_xor((int)most, 1));
  most = max(most, (unsigned)__shfl_xor((int)most, 2));
  // max = m 2^x with 1 <= m < 2: e = x - 2 where m <= 1.75, else x - 1; the sum carries into the exponent exactly then
  int e = (int)((most + 0x1FFFFFu) >> 23) - 2;
  e = min(max(e, 1), std::is_same<T, _Float16>::value ? 140 : 252);
  const float scale = __uint_as_float((unsigned)e << 23);
  unsigned w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
  *(unsigned*)(p.d_codes + slot * p.code_row + head * p.code_head + chunk * 4) = w;
  if ((chunk & 3) == 0) p.d_exps[slot * p.exp_row + head * p.exp_head + chunk / 4] = (uint8_t)(most >= 0x7F800000u ? 255 : e);
}

// A thread of the 16-bit types stores its chunk of both tensors: two loads in flight, one look at the slot (51200 tokens of 8 heads of 128, fp16:
// 75 -> 64 us); in fp32 a chunk is two loads already, and one thread per tensor is the faster (34 us : 35 for 29498 tokens of 8 heads of 64).
template <typename T>
__global__ __launch_bounds__(256) void cache4_store_kernel(Cache4Args a) {
  constexpr int BOTH = sizeof(T) == 2 ? 2 : 1;
  int k, tok, head, chunk;
  // the four lanes of a group come and go together: a group is one token and head
  if (!chunk_of(a, &k, &tok, &head, &chunk)) return;
  const long long slot = a.slots[tok];
  float v[BOTH][8];
#pragma unroll
  for (int i = 0; i < BOTH; ++i) read8((const T*)a.x[k + i] + (long long)tok * a.token[k + i] + (long long)head * a.head[k + i] + chunk * 8, v[i]);
  if (slot < 0 || slot >= a.rows) return;
#pragma unroll
  for (int i = 0; i < BOTH; ++i) store_group<T>(a.plane[k + i], v[i], slot, head, chunk);
}

template <typename T>
__global__ __launch_bounds__(256) void cache4_load_kernel(Cache4Args a) {
  int k, tok, head, chunk;
  if (!chunk_of(a, &k, &tok, &head, &chunk)) return;
  const long long slot = a.slots[tok];
  const bool in = slot >= 0 && slot < a.rows;
  const octo_cache4_plane& p = a.plane[k];
  const unsigned w = in ? *(const unsigned*)(p.d_codes + slot * p.code_row + head * p.code_head + chunk * 4) : 0u;
  const float scale = __uint_as_float(in ? (unsigned)p.d_exps[slot * p.exp_row + head * p.exp_head + chunk / 4] << 23 : 0x3F800000u);
  T* y = (T*)a.x[k] + (long long)tok * a.token[k] + (long long)head * a.head[k] + chunk * 8;
  if constexpr (sizeof(T) == 4) {
    typedef float floatx2 __attribute__((ext_vector_type(2)));
    const floatx2 f0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), f1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    const floatx2 f2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), f3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    __builtin_nontemporal_store(floatx4{f0[0], f0[1], f1[0], f1[1]}, (floatx4*)y);
    __builtin_nontemporal_store(floatx4{f2[0], f2[1], f3[0], f3[1]}, (floatx4*)(y + 4));
  } else {
    u32x4 o;
    if constexpr (std::is_same<T, _Float16>::value) {
      o[0] = __builtin_bit_cast(unsigned, (half2v)__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0));
      o[1] = __builtin_bit_cast(unsigned, (half2v)__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1));
      o[2] = __builtin_bit_cast(unsigned, (half2v)__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2));
      o[3] = __builtin_bit_cast(unsigned, (half2v)__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3));
    } else {
      o[0] = __builtin_bit_cast(unsigned, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
      o[1] = __builtin_bit_cast(unsigned, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
      o[2] = __builtin_bit_cast(unsigned, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
      o[3] = __builtin_bit_cast(unsigned, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    }
    __builtin_nontemporal_store(o, (u32x4*)y);
  }
}

bool plane_ok(const octo_cache4_plane& p) {
  return p.d_codes && p.d_exps && !((uintptr_t)p.d_codes & 15) && p.code_row >= 0 && p.code_head >= 0 && p.exp_row >= 0 && p.exp_head >= 0 &&
         !((p.code_row | p.code_head) & 15);
}

octo_status cache4_args(const octo_cache4_op* op, Cache4Args* a) {
  if (!op || (op->dtype != OCTO_F32 && op->dtype != OCTO_F16 && op->dtype != OCTO_BF16)) return OCTO_EINVAL;
  if (op->n < 0 || op->heads < 1 || op->rows < 1 || op->dim < 32 || op->dim > 128 || op->dim % 32 || !op->d_k || !op->d_v || !op->d_slots) return OCTO_EINVAL;
  if (!plane_ok(op->k_plane) || !plane_ok(op->v_plane) || op->k_token < 0 || op->k_head < 0 || op->v_token < 0 || op->v_head < 0) return OCTO_EINVAL;
  const int es = op->dtype == OCTO_F32 ? 4 : 2;
  if ((((uintptr_t)op->d_k | (uintptr_t)op->d_v) & 15) || ((op->k_token | op->k_head | op->v_token | op->v_head) * es & 15) || ((uintptr_t)op->d_slots & 7)) return OCTO_EINVAL;
  const long long total = (long long)op->n * op->heads * (op->dim / 8);
  if (total > 0x7FFFFF00ll) return OCTO_EINVAL;
  a->plane[0] = op->k_plane; a->plane[1] = op->v_plane;
  a->x[0] = op->d_k; a->x[1] = op->d_v; a->token[0] = op->k_token; a->token[1] = op->v_token; a->head[0] = op->k_head; a->head[1] = op->v_head;
  a->slots = (const long long*)op->d_slots; a->n_dyn = op->d_n; a->rows = op->rows; a->n = op->n; a->heads = op->heads;
  a->chunks = (unsigned)op->dim / 8; a->total = (unsigned)total;
  a->div_chunks = make_fastdiv(a->chunks); a->div_heads = make_fastdiv((unsigned)op->heads);
  return OCTO_OK;
}

const float E2M1[8] = {0.0f, 0.5f, 1.0f, 1.5f, 2.0f, 3.0f, 4.0f, 6.0f};

}  // namespace
}  // namespace octo

using namespace octo;

extern "C" {

octo_status octo_op_cache4_store(const octo_cache4_op* op, void* hip_stream) {
  Cache4Args a{};
  const octo_status st = cache4_args(op, &a);
  if (st != OCTO_OK || !a.total) return st;
  const dim3 grid((a.total + 255) / 256, op->dtype == OCTO_F32 ? 2 : 1);
  hipStream_t s = (hipStream_t)hip_stream;
  if (op->dtype == OCTO_F32) hipLaunchKernelGGL(cache4_store_kernel<float>, grid, dim3(256), 0, s, a);
  else if (op->dtype == OCTO_F16) hipLaunchKernelGGL(cache4_store_kernel<_Float16>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(cache4_store_kernel<__bf16>, grid, dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? OCTO_OK : OCTO_EHIP;
}

octo_status octo_op_cache4_load(const octo_cache4_op* op, void* hip_stream) {
  Cache4Args a{};
  const octo_status st = cache4_args(op, &a);
  if (st != OCTO_OK || !a.total) return st;
  const dim3 grid((a.total + 255) / 256, 2);
  hipStream_t s = (hipStream_t)hip_stream;
  if (op->dtype == OCTO_F32) hipLaunchKernelGGL(cache4_load_kernel<float>, grid, dim3(256), 0, s, a);
  else if (op->dtype == OCTO_F16) hipLaunchKernelGGL(cache4_load_kernel<_Float16>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(cache4_load_kernel<__bf16>, grid, dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? OCTO_OK : OCTO_EHIP;
}

octo_status octo_quantize_mx4(const float* src, size_t n, uint8_t* codes, uint8_t* exps) {
  if (n % 32 || ((!src || !codes || !exps) && n)) return OCTO_EINVAL;
  for (size_t g = 0; g < n / 32; ++g) {
    const float* x = src + 32 * g;
    float most = 0.f;
    bool finite = true;
    for (int i = 0; i < 32; ++i) { finite = finite && std::isfinite(x[i]); most = std::fmax(most, std::fabs(x[i])); }
    int e = -126;                                // the smallest exponent with most <= 7 * 2^e
    if (finite && most > 0.f) {
      int ex = 0;
      const float m = std::frexp(most, &ex);     // most = m * 2^ex, 0.5 <= m < 1
      e = m <= 0.875f ? ex - 3 : ex - 2;
      e = e < -126 ? -126 : e > 125 ? 125 : e;
    }
    exps[g] = finite ? (uint8_t)(e + 127) : 255;
    for (int i = 0; i < 32; ++i) {
      const double q = finite ? std::fabs(std::ldexp((double)x[i], -e)) : 0.0;
      int code = 0;                              // the nearest value, the even code in the middle between two
      while (code < 7) {
        const double mid = 0.5 * ((double)E2M1[code] + (double)E2M1[code + 1]);
        if (q < mid || (q == mid && code % 2 == 0)) break;
        ++code;
      }
      const uint8_t nib = (uint8_t)(code | (std::signbit(x[i]) ? 8 : 0));
      uint8_t* b = codes + 16 * g + i / 2;
      *b = i % 2 ? (uint8_t)(*b | nib << 4) : nib;
    }
  }
  return OCTO_OK;
}

octo_status octo_dequantize_mx4(const uint8_t* codes, const uint8_t* exps, size_t n, float* dst) {
  if (n % 32 || ((!codes || !exps || !dst) && n)) return OCTO_EINVAL;
  for (size_t i = 0; i < n; ++i) {
    const int c = codes[i / 2] >> (i % 2 ? 4 : 0) & 15;
    const float m = exps[i / 32] == 255 ? std::nanf("") : std::ldexp(E2M1[c & 7], exps[i / 32] - 127);
    dst[i] = c & 8 ? -m : m;
  }
  return OCTO_OK;
}

}  // extern "C"
