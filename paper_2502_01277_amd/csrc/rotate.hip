// octo_op_rotate: norm of every head and rotation by the token's positions, queries and keys in one launch.
//
// The bound is memory: every value is read and written once, against some ten operations.  The angles depend on the token and
// the pair alone, so a block of four wavefronts takes a few tokens, makes their cosines and sines once (one or two pairs a thread)
// in LDS and then walks over the heads of both tensors, 64 / lanes-per-head heads of one token per wavefront and step, four steps'
// loads at a time.  A lane holds VEC pairs, both elements of each: a rotation needs no exchange between lanes, a norm only
// the sum over the lanes of a head.
//
// An angle is pos * f / 2 pi revolutions.  The product is taken in fp64 and only its fraction goes to fp32 and to the sine and
// cosine instructions, whose argument is in revolutions (1.3e-7 off at most on [0, 1)): positions of any size lose nothing, where an fp32 angle at
// position 60000 is off by 4e-3.
#include <cmath>

#include "mfma_common.h"
#include "octo_internal.h"

namespace octo {
namespace {

struct RotateArgs {
  const void* x[2]; void* y[2]; const float* w[2];
  long long x_token[2], x_head[2], y_token[2], y_head[2];
  int heads0, heads;                 // heads of the first tensor, of both
  int n; const int* n_dyn;
  int dim, pairs, n_axes;            // pairs that are turned
  int split;                         // 0: interleaved
  int first[OCTO_MAX_AXES + 1];      // first pair of each axis, `pairs` behind the last
  int shared;
  double log2_base;
  const int* pos;
  float eps, inv_dim;
  int lanes;                         // per head, a power of two >= dim / 2 / VEC
  int steps;                         // per token: heads / (64 / lanes), rounded up
  int table;                         // pairs, rounded up to a power of two
  int tokens;                        // per block
};

template <typename T, int N> struct alignas(sizeof(T) * N) Pack { T v[N]; };

template <typename T, int VEC>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a) {
  constexpr int DEPTH = 4;
  __shared__ float2 turn[512];           // [token of the block][pair]
  __shared__ float weight[2][256];
  const int n = a.n_dyn ? min(max(*a.n_dyn, 0), a.n) : a.n;
  const int token0 = blockIdx.x * a.tokens;
  if (token0 >= n) return;
  const int here = min(a.tokens, n - token0);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int part_lane = lane & (a.lanes - 1), head_in_step = lane / a.lanes, per_step = 64 / a.lanes;
  const int half = a.dim / 2, p0 = part_lane * VEC;
  const bool works = p0 < half;
  // elements of the lane's pairs: VEC from i0 and VEC from i1 (split), or 2 VEC from i0
  int i0, i1;
  if (!a.split) { i0 = 2 * p0; i1 = i0 + VEC; }
  else if (p0 < a.pairs) { i0 = p0; i1 = p0 + a.pairs; }
  else { i0 = a.pairs + p0; i1 = i0 + half - a.pairs; }
  const int items = here * a.steps;
  typedef Pack<T, VEC> P;

  P in[DEPTH][2];
  auto place = [&](int item, int* tok, int* head) {
    *tok = item / a.steps;
    *head = (item - *tok * a.steps) * per_step + head_in_step;
    return works && item < items && *head < a.heads;
  };
  auto load = [&](int first_item) {
#pragma unroll
    for (int s = 0; s < DEPTH; ++s) {
      int tok, head;
      if (!place(first_item + 4 * s, &tok, &head)) continue;
      const int k = head >= a.heads0;
      const T* x = (const T*)a.x[k] + (long long)(token0 + tok) * a.x_token[k] + (long long)(head - (k ? a.heads0 : 0)) * a.x_head[k];
      in[s][0] = *(const P*)(x + i0);
      in[s][1] = *(const P*)(x + i1);
    }
  };
  load(wave);

  for (int i = threadIdx.x; i < 2 * a.dim; i += 256) {
    const int k = i >= a.dim, d = k ? i - a.dim : i;
    if (a.w[k]) weight[k][d] = a.w[k][d];
  }
  if (a.pairs) {
    const int p = threadIdx.x & (a.table - 1);
    int axis = 0;
    while (axis + 1 < a.n_axes && p >= a.first[axis + 1]) ++axis;
    const int count = a.shared ? a.pairs : a.first[axis + 1] - a.first[axis];
    const double f = exp2(-(double)(a.shared ? p : p - a.first[axis]) / count * a.log2_base) * 0.15915494309189533577;
    if (p < a.pairs)
      for (int t = threadIdx.x / a.table; t < here; t += 256 / a.table) {
        const double rev = (double)a.pos[(size_t)(token0 + t) * a.n_axes + axis] * f;
        const float r = (float)(rev - floor(rev));
        turn[t * a.table + p] = make_float2(__builtin_amdgcn_cosf(r), __builtin_amdgcn_sinf(r));
      }
  }
  __syncthreads();

  for (int first_item = wave; first_item < items; first_item += 4 * DEPTH) {
    if (first_item != wave) load(first_item);
#pragma unroll
    for (int s = 0; s < DEPTH; ++s) {
      int tok, head;
      const bool any = place(first_item + 4 * s, &tok, &head);
      if (first_item + 4 * s >= items) break;                     // the same for the whole wavefront
      const int k = any && head >= a.heads0;
      float u[2 * VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) { u[e] = any ? (float)in[s][0].v[e] : 0.f; u[VEC + e] = any ? (float)in[s][1].v[e] : 0.f; }
      if (a.w[0] || a.w[1]) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) sum += u[e] * u[e];
        for (int d = 1; d < a.lanes; d *= 2) sum += __shfl_xor(sum, d);
        if (a.w[k]) {
          const float r = 1.0f / sqrtf(sum * a.inv_dim + a.eps);
          if (works) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) { u[e] *= r * weight[k][i0 + e]; u[VEC + e] *= r * weight[k][i1 + e]; }
          }
        }
      }
      if (!any) continue;
      if (p0 < a.pairs) {
        const float2* c = turn + tok * a.table + p0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const int first = a.split ? e : 2 * e, second = a.split ? VEC + e : 2 * e + 1;
          if (p0 + e < a.pairs) {
            const float2 t = c[e];
            const float x1 = u[first], x2 = u[second];
            u[first] = x1 * t.x - x2 * t.y;
            u[second] = x2 * t.x + x1 * t.y;
          }
        }
      }
      T* y = (T*)a.y[k] + (long long)(token0 + tok) * a.y_token[k] + (long long)(head - (k ? a.heads0 : 0)) * a.y_head[k];
      P o0, o1;
#pragma unroll
      for (int e = 0; e < VEC; ++e) { o0.v[e] = (T)u[e]; o1.v[e] = (T)u[VEC + e]; }
      *(P*)(y + i0) = o0;
      *(P*)(y + i1) = o1;
    }
  }
}

template <typename T, int VEC>
hipError_t launch_vec(const RotateArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((rotate_kernel<T, VEC>), dim3((a.n + a.tokens - 1) / a.tokens), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_type(int vec, const RotateArgs& a, hipStream_t s) {
  if constexpr (sizeof(T) == 2) if (vec == 8) return launch_vec<T, 8>(a, s);
  if (vec == 4) return launch_vec<T, 4>(a, s);
  if (vec == 2) return launch_vec<T, 2>(a, s);
  return launch_vec<T, 1>(a, s);
}

}  // namespace
}  // namespace octo

using namespace octo;

extern "C" octo_status octo_op_rotate(const octo_rotate_op* op, void* hip_stream) {
  if (!op || (op->dtype != OCTO_F32 && op->dtype != OCTO_F16 && op->dtype != OCTO_BF16)) return OCTO_EINVAL;
  if (op->n_tokens < 0 || op->dim < 2 || op->dim > 256 || op->dim % 2 || op->n_axes < 0 || op->n_axes > OCTO_MAX_AXES || op->n_parts < 1 || op->n_parts > OCTO_MAX_ROTATE_PARTS) return OCTO_EINVAL;
  if (op->pairs < OCTO_PAIRS_SPLIT || op->pairs > OCTO_PAIRS_INTERLEAVED || op->ladder < OCTO_LADDER_AXIS || op->ladder > OCTO_LADDER_SHARED) return OCTO_EINVAL;
  if (op->n_axes && (!op->d_pos || !(op->base > 0) || !std::isfinite(op->base) || ((uintptr_t)op->d_pos & 3))) return OCTO_EINVAL;
  RotateArgs a{};
  const int es = op->dtype == OCTO_F32 ? 4 : 2, half = op->dim / 2;
  for (int i = 0; i < op->n_axes; ++i) {
    if (op->sections[i] < 0 || op->sections[i] > half) return OCTO_EINVAL;
    a.first[i + 1] = a.first[i] + op->sections[i];
  }
  a.pairs = a.first[op->n_axes];
  if (a.pairs > half) return OCTO_EINVAL;
  a.n_axes = op->n_axes; a.n = op->n_tokens; a.n_dyn = op->d_n; a.dim = op->dim; a.pos = op->d_pos; a.eps = op->eps; a.inv_dim = 1.0f / (float)op->dim;
  a.split = op->pairs == OCTO_PAIRS_SPLIT; a.shared = op->ladder == OCTO_LADDER_SHARED; a.log2_base = op->n_axes ? std::log2(op->base) : 0.0;
  // what the vectors have to divide: counts of elements, and all addresses in elements
  unsigned long long align = a.split ? (unsigned)(a.pairs | (half - a.pairs)) : (unsigned)half;
  for (int k = 0; k < op->n_parts; ++k) {
    const octo_rotate_part& p = op->part[k];
    if (!p.d_x || !p.d_y || p.heads < 1 || p.heads > 65536 || p.x_token < 0 || p.x_head < 0 || p.y_token < 0 || p.y_head < 0) return OCTO_EINVAL;
    if (p.d_weight && !(op->eps >= 0)) return OCTO_EINVAL;
    if (((uintptr_t)p.d_x | (uintptr_t)p.d_y) % es || ((uintptr_t)p.d_weight & 3)) return OCTO_EINVAL;
    align |= (uintptr_t)p.d_x / es | (uintptr_t)p.d_y / es | (unsigned long long)(p.x_token | p.x_head | p.y_token | p.y_head);
    a.x[k] = p.d_x; a.y[k] = p.d_y; a.w[k] = p.d_weight;
    a.x_token[k] = p.x_token; a.x_head[k] = p.x_head; a.y_token[k] = p.y_token; a.y_head[k] = p.y_head;
    if (!k) a.heads0 = p.heads;
    a.heads += p.heads;
  }
  int vec = 16 / es;
  while (vec > 1 && align % vec) vec /= 2;
  if (half > 64 * vec) return OCTO_EINVAL;
  a.lanes = 1;
  while (a.lanes * vec < half) a.lanes *= 2;
  a.steps = (a.heads + 64 / a.lanes - 1) / (64 / a.lanes);
  a.table = 1;
  while (a.table < a.pairs) a.table *= 2;
  // Tokens of a block: as many as give each wavefront two rounds of loads, unless that leaves fewer than eight blocks per compute unit.
  const int most = 512 / a.table < 16 ? 512 / a.table : 16;
  a.tokens = (32 + a.steps - 1) / a.steps;
  if (a.tokens > most) a.tokens = most;
  while (a.tokens > 1 && (op->n_tokens + a.tokens - 1) / a.tokens < 2048) a.tokens = (a.tokens + 1) / 2;
  if (op->n_tokens == 0) return OCTO_OK;
  hipStream_t s = (hipStream_t)hip_stream;
  const hipError_t e = op->dtype == OCTO_F32 ? launch_type<float>(vec, a, s) : op->dtype == OCTO_F16 ? launch_type<_Float16>(vec, a, s) : launch_type<__bf16>(vec, a, s);
  return e == hipSuccess ? OCTO_OK : OCTO_EHIP;
}
