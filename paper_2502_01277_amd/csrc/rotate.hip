// octo_op_rotate: norm of every head and rotation by the token's positions, queries and keys in one launch.
//
// The bound is memory: every value is read and written once, against some ten operations.  The heads of both tensors and all tokens are one
// list of rows; a lane holds VEC pairs of a row, both elements of each (a rotation then needs no exchange between lanes, a norm only the sum over
// the lanes of a row), a wavefront as many rows at a time as its lanes hold, and it walks over `items` such groups with the
// loads of four in flight.  The angles depend on token and pair alone: the wavefront makes the cosines and sines of its few tokens
// once, in LDS, while its first loads are on their way.  Wavefronts are independent of each other.
//
// An angle is pos * f / 2 pi revolutions.  The product is taken in fp64 and only its fraction goes to fp32 and to the sine and
// cosine instructions, whose argument is in revolutions (1.3e-7 off at most on [0, 1)): positions of any size lose nothing, where an fp32 angle at
// position 60000 is off by 4e-3.
#include <cmath>

#include "mfma_common.h"
#include "octo_internal.h"

namespace octo {
namespace {

constexpr int TURNS = 512;           // cosines and sines a wavefront can hold

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
  int w_aligned;                     // weights on 16 bytes
  int lanes, rows;                   // per row: dim / 2 / VEC; rows at a time: 64 / lanes
  int items;                         // groups of rows of a wavefront
  int table;                         // pairs, rounded up to a power of two
  unsigned total;                    // rows in all
  int blocks;                        // to start
  FastDiv div_heads, div_lanes;
};

template <typename T, int N> struct alignas(sizeof(T) * N) Pack { T v[N]; };
// Results go past the caches' reuse order: nothing here reads them again (51200 tokens of 32 + 8 heads of 128, bf16: 255 -> 246 us; 300
// regions of 49 tokens, 8 + 8 heads of 64, fp16: 18.0 -> 16.8; the same for loads made it slower).
template <typename P> __device__ __forceinline__ void store_once(P* p, const P& v) {
  if constexpr (sizeof(P) == 16) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4*)p);
  else *p = v;
}

// Sum over the lanes of a row, the same in each; `at` is the lane's place in its row.
__device__ __forceinline__ float row_sum(float v, int lanes, int at, int lane) {
  if ((lanes & (lanes - 1)) == 0) {
    for (int d = 1; d < lanes; d *= 2) v += __shfl_xor(v, d);
    return v;
  }
  for (int left = lanes; left > 1;) {
    const int h = (left + 1) / 2;
    const float o = __shfl(v, (lane + h) & 63);
    if (at + h < left) v += o;
    left = h;
  }
  return __shfl(v, lane - at);
}

template <typename T, int VEC>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a) {
  constexpr int DEPTH = 4;
  __shared__ float2 turns[4][TURNS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float2* const turn = turns[wave];                     // [token of the wavefront][pair]
  const unsigned total = a.n_dyn ? (unsigned)min(max(*a.n_dyn, 0), a.n) * (unsigned)a.heads : a.total;
  const unsigned per_wave = (unsigned)(a.items * a.rows), r0 = (blockIdx.x * 4 + wave) * per_wave;
  if (r0 >= total) return;
  const unsigned r_end = min(total, r0 + per_wave);
  const int row_of_lane = (int)fast_div((unsigned)lane, a.div_lanes), at = lane - row_of_lane * a.lanes;
  const int half = a.dim / 2, p0 = at * VEC;
  const bool works = row_of_lane < a.rows;
  // elements of the lane's pairs: VEC from i0 and VEC from i1 (split), or 2 VEC from i0
  int i0, i1;
  if (!a.split) { i0 = 2 * p0; i1 = i0 + VEC; }
  else if (p0 < a.pairs) { i0 = p0; i1 = p0 + a.pairs; }
  else { i0 = a.pairs + p0; i1 = i0 + half - a.pairs; }
  typedef Pack<T, VEC> P;

  P in[DEPTH][2];
  auto load = [&](unsigned first) {
#pragma unroll
    for (int s = 0; s < DEPTH; ++s) {
      const unsigned r = first + s * a.rows + row_of_lane;
      if (!works || r >= r_end) continue;
      const unsigned tok = fast_div(r, a.div_heads);
      int head = (int)(r - tok * (unsigned)a.heads);
      const int k = head >= a.heads0;
      head -= k ? a.heads0 : 0;
      const T* x = (const T*)a.x[k] + tok * a.x_token[k] + head * a.x_head[k];
      in[s][0] = *(const P*)(x + i0);
      in[s][1] = *(const P*)(x + i1);
    }
  };
  load(r0);

  const unsigned tok0 = fast_div(r0, a.div_heads);
  const int tokens = (int)(fast_div(r_end - 1, a.div_heads) - tok0) + 1;
  for (int p = lane & (a.table - 1); p < a.pairs; p += 64) {
    int axis = 0;
    while (axis + 1 < a.n_axes && p >= a.first[axis + 1]) ++axis;
    const int count = a.shared ? a.pairs : a.first[axis + 1] - a.first[axis], step = a.table < 64 ? 64 / a.table : 1;
    const double f = exp2(-(double)(a.shared ? p : p - a.first[axis]) / count * a.log2_base) * 0.15915494309189533577;
    for (int t = a.table < 64 ? lane / a.table : 0; t < tokens; t += step) {
      const double rev = (double)a.pos[(size_t)(tok0 + t) * a.n_axes + axis] * f;
      const float r = (float)(rev - floor(rev));
      turn[t * a.pairs + p] = make_float2(__builtin_amdgcn_cosf(r), __builtin_amdgcn_sinf(r));
    }
  }
  float weight[2][2 * VEC];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (!a.w[k]) continue;                              // not used then
    const float* w0 = a.w[k] + (works ? i0 : 0);
    const float* w1 = a.w[k] + (works ? i1 : 0);
    if (VEC % 4 == 0 && a.w_aligned) {
#pragma unroll
      for (int e = 0; e < VEC; e += 4) {
        const floatx4 f0 = *(const floatx4*)(w0 + e), f1 = *(const floatx4*)(w1 + e);
#pragma unroll
        for (int c = 0; c < 4; ++c) { weight[k][e + c] = f0[c]; weight[k][VEC + e + c] = f1[c]; }
      }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) { weight[k][e] = w0[e]; weight[k][VEC + e] = w1[e]; }
    }
  }
  // the cosines and sines are read by other lanes of this wavefront: its LDS accesses stay in order
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");

  for (unsigned first = r0; first < r_end; first += DEPTH * a.rows) {
    if (first != r0) load(first);
#pragma unroll
    for (int s = 0; s < DEPTH; ++s) {
      if (first + s * a.rows >= r_end) break;                     // the same for the whole wavefront
      const unsigned r = first + s * a.rows + row_of_lane;
      const bool any = works && r < r_end;
      const unsigned tok = fast_div(any ? r : r0, a.div_heads);
      int head = any ? (int)(r - tok * (unsigned)a.heads) : 0;
      const int k = head >= a.heads0;
      head -= k ? a.heads0 : 0;
      float u[2 * VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) { u[e] = any ? (float)in[s][0].v[e] : 0.f; u[VEC + e] = any ? (float)in[s][1].v[e] : 0.f; }
      if (a.w[0] || a.w[1]) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) sum += u[e] * u[e];
        sum = row_sum(sum, a.lanes, at, lane);
        const float f = 1.0f / sqrtf(sum * a.inv_dim + a.eps);
        if (k ? a.w[1] : a.w[0]) {
#pragma unroll
          for (int e = 0; e < 2 * VEC; ++e) u[e] *= f * (k ? weight[1][e] : weight[0][e]);
        }
      }
      if (!any) continue;
      if (p0 < a.pairs) {
        const float2* c = turn + (tok - tok0) * a.pairs + p0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          if (p0 + e < a.pairs) {
            const float2 t = c[e];
            const float x1 = a.split ? u[e] : u[2 * e], x2 = a.split ? u[VEC + e] : u[2 * e + 1];
            const float y1 = x1 * t.x - x2 * t.y, y2 = x2 * t.x + x1 * t.y;
            if (a.split) { u[e] = y1; u[VEC + e] = y2; } else { u[2 * e] = y1; u[2 * e + 1] = y2; }
          }
        }
      }
      T* y = (T*)a.y[k] + tok * a.y_token[k] + head * a.y_head[k];
      P o0, o1;
#pragma unroll
      for (int e = 0; e < VEC; ++e) { o0.v[e] = (T)u[e]; o1.v[e] = (T)u[VEC + e]; }
      store_once((P*)(y + i0), o0);
      store_once((P*)(y + i1), o1);
    }
  }
}

template <typename T, int VEC>
hipError_t launch_vec(const RotateArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((rotate_kernel<T, VEC>), dim3((unsigned)a.blocks), dim3(256), 0, s, a);
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
    a.w_aligned = (k == 0 || a.w_aligned) && ((uintptr_t)p.d_weight & 15) == 0;
    a.x[k] = p.d_x; a.y[k] = p.d_y; a.w[k] = p.d_weight;
    a.x_token[k] = p.x_token; a.x_head[k] = p.x_head; a.y_token[k] = p.y_token; a.y_head[k] = p.y_head;
    if (!k) a.heads0 = p.heads;
    a.heads += p.heads;
  }
  int vec = 16 / es;
  while (vec > 1 && align % vec) vec /= 2;
  if (half > 64 * vec) return OCTO_EINVAL;
  a.lanes = half / vec;
  a.rows = 64 / a.lanes;
  a.table = 1;
  while (a.table < a.pairs) a.table *= 2;
  const unsigned long long total = (unsigned long long)op->n_tokens * a.heads;
  if (total > 0x7FFF0000ull) return OCTO_EINVAL;
  a.total = (unsigned)total;
  a.div_heads = make_fastdiv((unsigned)a.heads); a.div_lanes = make_fastdiv((unsigned)a.lanes);
  // Groups of rows a wavefront: up to eight, as long as that leaves 4096 wavefronts and its tokens' turns fit (one group's always do).
  const unsigned long long groups = (total + a.rows - 1) / a.rows;
  a.items = groups / 4096 < 1 ? 1 : groups / 4096 > 8 ? 8 : (int)(groups / 4096);
  while (a.items > 1 && ((a.items * a.rows + a.heads - 2) / a.heads + 1) * a.pairs > TURNS) --a.items;
  const unsigned long long blocks = (total + 4ull * a.items * a.rows - 1) / (4ull * a.items * a.rows);
  if (blocks > 0xFFFFFF) return OCTO_EINVAL;                // HIP counts the threads of a launch, 256 a block, in 32 bits
  a.blocks = (int)blocks;
  if (op->n_tokens == 0) return OCTO_OK;
  hipStream_t s = (hipStream_t)hip_stream;
  const hipError_t e = op->dtype == OCTO_F32 ? launch_type<float>(vec, a, s) : op->dtype == OCTO_F16 ? launch_type<_Float16>(vec, a, s) : launch_type<__bf16>(vec, a, s);
  return e == hipSuccess ? OCTO_OK : OCTO_EHIP;
}
