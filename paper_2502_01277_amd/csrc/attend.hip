// octo_op_attend: arguments, and the kernel that joins parts.
#include <algorithm>
#include <cmath>
#include <mutex>

#include "attend_tile.h"

namespace octo {
namespace {

// Adds up the parts of a row: sum_p 2^(ref_p - m) (o_p, sum_p), m the largest reference, in the order of the parts.  Half a wavefront has a
// row: its lanes take references and sums of 32 parts at a time, then four elements of dim each.
template <typename T>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  Span sp;
  const unsigned rows8 = fast_div(blockIdx.x, a.div_seq);             // neighbours: the same rows of different sequences
  if (!span_of(a, (int)(blockIdx.x - rows8 * (unsigned)a.n_seq), &sp)) return;
  const int parts = parts_of(sp.n_kv, a.cut ? even_part(sp.n_kv, *a.cut_tiles) : a.part_keys), r = (int)rows8 * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31, d = lane * 4;
  if (parts == 1 || r >= sp.n_q * a.q_heads) return;
  const long long at = (long long)sp.q0 * a.q_heads + r, step = (long long)a.n_q * a.q_heads;
  // the first parts' sums are on their way while the references are compared; memory of all n_split parts is there, used or not
  constexpr int AHEAD = 8;
  const float* y = a.part_o + at * a.dim + (d < a.dim ? d : 0);
  floatx4 held[AHEAD];
#pragma unroll
  for (int p = 0; p < AHEAD; ++p) held[p] = *(const floatx4*)(y + (p < parts ? p : 0) * step * a.dim);
  float2 x[MAX_PARTS / 32];
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < MAX_PARTS / 32; ++k) {
    x[k] = 32 * k + lane < parts ? a.part_ml[at + (32 * k + lane) * step] : make_float2(-INFINITY, 0.f);
    m = fmaxf(m, x[k].x);
  }
  for (int i = 1; i < 32; i *= 2) m = fmaxf(m, __shfl_xor(m, i, 32));
  float total = 0.f;
#pragma unroll
  for (int k = 0; k < MAX_PARTS / 32; ++k) {
    x[k].x = x[k].x == m ? 1.0f : __builtin_amdgcn_exp2f(x[k].x - m);
    total += x[k].y * x[k].x;
  }
  for (int i = 1; i < 32; i *= 2) total += __shfl_xor(total, i, 32);
  floatx4 o = {0, 0, 0, 0};
#pragma unroll
  for (int p = 0; p < AHEAD; ++p) {
    const float f = __shfl(x[0].x, p, 32);
    if (p < parts) o += held[p] * f;
  }
  for (int p0 = AHEAD; p0 < parts; p0 += AHEAD) {
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) held[p] = *(const floatx4*)(y + (p0 + p < parts ? p0 + p : 0) * step * a.dim);
    const float w = p0 < 32 ? x[0].x : p0 < 64 ? x[1].x : p0 < 96 ? x[2].x : x[3].x;
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) {
      const float f = __shfl(w, (p0 + p) & 31, 32);
      if (p0 + p < parts) o += held[p] * f;
    }
  }
  if (d >= a.dim) return;
  const float inv = total != 0.f ? 1.0f / total : 0.f;
  if (d == 0 && a.lse) a.lse[at] = total != 0.f ? (m + log2f(total)) * 0.693147180559945f : -INFINITY;
  const int qi = r / a.q_heads, head = r - qi * a.q_heads;
  store4<T>((T*)a.out + (sp.q0 + (long long)qi) * a.out_row + head * a.out_head + d, o * inv);
}

constexpr int MAX_DEVICES = 64;
int cu_count() {
  static std::mutex mu;
  static int cus[MAX_DEVICES] = {};
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) return 0;
  std::lock_guard<std::mutex> lock(mu);
  if (!cus[dev]) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 0;
    cus[dev] = n;
  }
  return cus[dev];
}

bool sizes_ok(const octo_attend_op* op) {
  if (!op || op->dtype < OCTO_F32 || op->dtype > OCTO_BF16 || op->kv_format < OCTO_KV_PLAIN || op->kv_format > OCTO_KV_CACHE4) return false;
  if (op->kv_format == OCTO_KV_CACHE4 && op->dtype == OCTO_F32) return false;
  if (op->dim < 8 || op->dim > 128 || op->dim % (op->kv_format == OCTO_KV_CACHE4 ? 32 : 8)) return false;
  if (op->kv_heads < 1 || op->q_heads < op->kv_heads || op->q_heads % op->kv_heads || op->q_heads > 4096) return false;
  if (op->n_seq < 0 || op->n_q < 0 || op->max_q < 0 || op->max_kv < 0 || op->kv_rows < 0) return false;
  if (op->max_q > op->n_q || op->max_kv > 0x7FFFFF00) return false;
  if ((long long)op->max_q * op->q_heads > 0x7FFFFF00) return false;       // rows of a sequence are numbered in 31 bits
  return (double)op->n_seq * op->kv_heads * (op->max_q * (double)(op->q_heads / op->kv_heads) / 16 + 1) < 2e9;
}
size_t part_bytes(const octo_attend_op* op, const Plan& p) {
  return p.n_split > 1 ? (size_t)p.n_split * op->n_q * op->q_heads * ((size_t)op->dim * 4 + 8) + 16 : 0;
}
bool stride_ok(long long elems, int es) { return elems >= 0 && (elems * es & 15) == 0; }
constexpr long long MOST_ROW = 16 << 20;      // bytes between rows: 32 of them stay inside a buffer's 31 bits

}  // namespace
}  // namespace octo

using namespace octo;

extern "C" {

size_t octo_op_attend_workspace_bytes(const octo_attend_op* op) {
  if (!sizes_ok(op) || !op->n_seq || !op->max_q) return 0;
  const int cus = cu_count();
  const Plan p = plan_of(op, cus > 0 ? cus : 256);
  return launch_blocks(op, p) > MOST_BLOCKS ? 0 : part_bytes(op, p);
}

octo_status octo_op_attend(const octo_attend_op* op, void* hip_stream, int32_t* kernel_id) {
  if (!sizes_ok(op) || !std::isfinite(op->scale) || !(op->scale > 0)) return OCTO_EINVAL;
  const int es = op->dtype == OCTO_F32 ? 4 : 2;
  if (!op->d_q || !op->d_out || !op->d_q_start || !op->d_kv_start || !op->d_kv_len) return OCTO_EINVAL;
  if ((((uintptr_t)op->d_q | (uintptr_t)op->d_out) & 15) || (((uintptr_t)op->d_q_start | (uintptr_t)op->d_kv_len | (uintptr_t)op->d_n_seq | (uintptr_t)op->d_lse) & 3) || ((uintptr_t)op->d_kv_start & 7)) return OCTO_EINVAL;
  if (!stride_ok(op->q_row, es) || !stride_ok(op->q_head, es) || !stride_ok(op->out_row, es) || !stride_ok(op->out_head, es)) return OCTO_EINVAL;
  AttendArgs a{};
  if (op->kv_format == OCTO_KV_PLAIN) {
    if ((op->kv_rows && (!op->d_k || !op->d_v)) || (((uintptr_t)op->d_k | (uintptr_t)op->d_v) & 15)) return OCTO_EINVAL;
    if (!stride_ok(op->k_row, es) || !stride_ok(op->k_head, es) || !stride_ok(op->v_row, es) || !stride_ok(op->v_head, es)) return OCTO_EINVAL;
    a.k = (const char*)op->d_k; a.v = (const char*)op->d_v;
    a.k_row = op->k_row * es; a.k_head = op->k_head * es; a.v_row = op->v_row * es; a.v_head = op->v_head * es;
  } else {
    const octo_cache4_plane* planes[2] = {&op->k_plane, &op->v_plane};
    for (const octo_cache4_plane* p : planes)
      if ((op->kv_rows && (!p->d_codes || !p->d_exps)) || ((uintptr_t)p->d_codes & 15) || !stride_ok(p->code_row, 1) || !stride_ok(p->code_head, 1) || p->exp_row < 0 || p->exp_head < 0 || p->exp_row >= MOST_ROW) return OCTO_EINVAL;
    a.k = (const char*)op->k_plane.d_codes; a.v = (const char*)op->v_plane.d_codes; a.k_exp = op->k_plane.d_exps; a.v_exp = op->v_plane.d_exps;
    a.k_row = op->k_plane.code_row; a.k_head = op->k_plane.code_head; a.v_row = op->v_plane.code_row; a.v_head = op->v_plane.code_head;
    a.ke_row = op->k_plane.exp_row; a.ke_head = op->k_plane.exp_head; a.ve_row = op->v_plane.exp_row; a.ve_head = op->v_plane.exp_head;
  }
  if (a.k_row >= MOST_ROW || a.v_row >= MOST_ROW) return OCTO_EINVAL;
  if (kernel_id) *kernel_id = 0;
  if (!op->n_seq || !op->max_q) return OCTO_OK;
  const int cus = cu_count();
  const Plan p = plan_of(op, cus > 0 ? cus : 256);
  const long long blocks = launch_blocks(op, p);
  if (blocks > MOST_BLOCKS) return OCTO_EINVAL;
  if (cus < 1) return OCTO_EHIP;
  const size_t need = part_bytes(op, p);
  if (need && (!op->d_workspace || ((uintptr_t)op->d_workspace & 15))) return OCTO_EINVAL;
  if (need > op->workspace_bytes) return OCTO_ENOMEM;
  a.q = op->d_q; a.q_row = op->q_row; a.q_head = op->q_head;
  a.q_start = op->d_q_start; a.kv_start = (const long long*)op->d_kv_start; a.kv_len = op->d_kv_len; a.n_dyn = op->d_n_seq; a.mask = op->d_key_mask;
  a.out = op->d_out; a.out_row = op->out_row; a.out_head = op->out_head; a.lse = op->d_lse;
  a.kv_rows = op->kv_rows; a.n_seq = op->n_seq; a.n_q = op->n_q; a.max_q = op->max_q; a.max_kv = op->max_kv; a.dim = op->dim;
  a.q_heads = op->q_heads; a.kv_heads = op->kv_heads; a.group = op->q_heads / op->kv_heads; a.div_group = make_fastdiv((unsigned)a.group);
  a.scale2 = op->scale * 1.44269504088896341f;
  a.n_split = p.n_split;
  if (need) {
    a.part_o = (float*)op->d_workspace;
    a.part_ml = (float2*)(a.part_o + (size_t)p.n_split * op->n_q * op->q_heads * op->dim);
    a.cut_tiles = (int*)(a.part_ml + (size_t)p.n_split * op->n_q * op->q_heads);
  }
  hipStream_t s = (hipStream_t)hip_stream;
  a.part_keys = p.part_keys;
  a.cut = p.cut; a.even_tiles = p.even_tiles;
  a.slots = p.slots;
  a.row_blocks = p.row_blocks;
  a.by_die = by_die(p, (long long)op->n_seq * op->kv_heads * p.n_split);
  a.blocks = (int)blocks;
  a.div_heads = make_fastdiv((unsigned)op->kv_heads); a.div_blocks = make_fastdiv((unsigned)p.row_blocks); a.div_split = make_fastdiv((unsigned)p.n_split);
  hipError_t e = p.kernel == TILES ? (op->dtype == OCTO_F16 ? launch_attend_tile_f16(op->kv_format, a, s) : launch_attend_tile_bf16(op->kv_format, a, s))
               : op->dtype == OCTO_F32 ? launch_attend_direct_f32(op->kv_format, p.how, a, s)
               : op->dtype == OCTO_F16 ? launch_attend_direct_f16(op->kv_format, p.how, a, s)
                                       : launch_attend_direct_bf16(op->kv_format, p.how, a, s);
  if (e == hipSuccess && p.n_split > 1) {
    a.div_seq = make_fastdiv((unsigned)op->n_seq);
    const dim3 grid((unsigned)join_blocks(op));
    if (op->dtype == OCTO_F32) hipLaunchKernelGGL(attend_join_kernel<float>, grid, dim3(256), 0, s, a);
    else if (op->dtype == OCTO_F16) hipLaunchKernelGGL(attend_join_kernel<_Float16>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(attend_join_kernel<__bf16>, grid, dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  if (kernel_id && e == hipSuccess) *kernel_id = 1000 * (p.how == DIRECT_SHARE2 ? 4 : p.cut ? 5 : p.kernel) + p.n_split;
  return e == hipSuccess ? OCTO_OK : OCTO_EHIP;
}

}  // extern "C"
