// octo_op_attend: what its kernels share, and the kernel whose wavefronts read keys and values straight from memory.
//
// Rows.  The queries of a sequence that read one key head, q_len x (q_heads / kv_heads) of them, are the rows of one product: a row r is
// query r / group of the sequence and head r % group of the group, so a key is read once for all of them.
//
// Products.  Scores are computed transposed, S^T = K Q^T: a lane then holds scores of ONE row (lane % 16) and of 8 of 32 keys, and the same lane
// needs, as the operand P^T of O^T = V^T P^T, eight weights of that row.  Which keys the eight slots of an operand stand for does
// not matter as long as V's operand has them in the same order, so slot j of lane group g is key 4 g + j (j < 4) or 16 + 4 g + j - 4: the weights
// go from one product to the other without leaving their registers.
#pragma once
#include <cfloat>

#include "attend_choice.h"
#include "mfma_common.h"

namespace octo {

struct AttendArgs {
  const void* q; long long q_row, q_head;                              // elements
  const char* k; const char* v; long long k_row, k_head, v_row, v_head;      // bytes, as all that follow
  const uint8_t* k_exp; const uint8_t* v_exp; long long ke_row, ke_head, ve_row, ve_head;
  const int* q_start; const long long* kv_start; const int* kv_len; const int* n_dyn;
  const uint8_t* mask;
  void* out; long long out_row, out_head;                              // elements
  float* lse;
  float* part_o; float2* part_ml;                                      // [part][row of q][head]: sums (dim floats each) and (reference, sum of weights)
  long long kv_rows;
  int n_seq, n_q, max_q, max_kv, dim, q_heads, kv_heads, group;
  FastDiv div_group;
  float scale2;                                                        // scale * log2(e)
  int n_split, part_keys;                                              // parts of part_keys keys (a multiple of 64); sequences of one part are finished by its block
  int row_blocks;                                                      // of the kernel's rows, of the longest sequence
  FastDiv div_heads, div_blocks, div_split, div_seq;                   // kv_heads, row_blocks, n_split, n_seq (the join's)
  int by_die;                                                          // blocks that read the same keys run on one die
  int even_tiles;                                                      // what cut takes as the length of a part where all sequences are alike, 0: nothing
  int blocks;                                                          // to start
  int cut, slots;                                                      // cut: attend_tile_kernel cuts its pieces itself, for so many blocks at a time;
  int* cut_tiles;                                                      // what it took as the length of a part, for attend_join_kernel
};

enum { KV_PLAIN = OCTO_KV_PLAIN, KV_CACHE4 = OCTO_KV_CACHE4 };

hipError_t launch_attend_direct_f16(int format, int how, const AttendArgs& a, hipStream_t s);
hipError_t launch_attend_direct_bf16(int format, int how, const AttendArgs& a, hipStream_t s);
hipError_t launch_attend_direct_f32(int format, int how, const AttendArgs& a, hipStream_t s);

#ifdef __HIPCC__
typedef uint32_t u32x3 __attribute__((ext_vector_type(3)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// The n-th piece of work.  Blocks of rows that read the same keys come one after the other, on one die (every eighth block runs there) where
// the sets of keys share out evenly over the eight, so that its cache has the keys for all of them; then come key heads, parts, and sequences last: neighbours are
// alike in length, and a short sequence's pieces do not all leave the same units idle.
struct Piece { int seq, part, block, head; };
__device__ __forceinline__ Piece piece_of(const AttendArgs& a, unsigned n, bool by_die) {
  Piece p;
  const unsigned q = by_die ? n >> 3 : n, r = fast_div(q, a.div_blocks);
  const unsigned w = by_die ? r * 8 + (n & 7) : r, y = fast_div(w, a.div_heads), z = fast_div(y, a.div_split);
  p.block = (int)(q - r * (unsigned)a.row_blocks); p.head = (int)(w - y * (unsigned)a.kv_heads); p.part = (int)(y - z * (unsigned)a.n_split); p.seq = (int)z;
  return p;
}
struct Span { int q0, n_q, n_kv; long long kv0; };
// The rows and keys of sequence b, cut to what the host stated; false: no such sequence, or no queries.
__device__ __forceinline__ bool span_of(const AttendArgs& a, int b, Span* s) {
  if (a.n_dyn && b >= *a.n_dyn) return false;
  const int lo = min(max(a.q_start[b], 0), a.n_q), hi = min(max(a.q_start[b + 1], lo), a.n_q);
  s->q0 = lo; s->n_q = min(hi - lo, a.max_q);
  const long long k0 = a.kv_start[b];
  const bool inside = k0 >= 0 && k0 < a.kv_rows;
  s->kv0 = inside ? k0 : 0;
  const long long room = inside ? a.kv_rows - k0 : 0;
  const int want = min(max(a.kv_len[b], 0), a.max_kv);
  s->n_kv = want < room ? want : (int)room;
  return s->n_q > 0;
}

// Eight operand values of a lane.
template <typename T> struct Eight { u32x4 v; };
template <> struct Eight<float> { floatx4 lo, hi; };
// C += A B for 16 x 16 and 32 of K; in fp32 as eight products of 4 of K, the j-th with every lane's value j.
template <typename T> __device__ __forceinline__ floatx4 mma(const Eight<T>& a, const Eight<T>& b, floatx4 c) {
  if constexpr (sizeof(T) == 2) {
    return mfma16<T>(a.v, b.v, c);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.lo[j], b.lo[j], c, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.hi[j], b.hi[j], c, 0, 0, 0);
    return c;
  }
}
template <typename T> __device__ __forceinline__ Eight<T> eight_of(floatx4 lo, floatx4 hi) {
  if constexpr (sizeof(T) == 2) {
    Eight<T> e;
    store4<T>((T*)&e.v, lo);
    store4<T>((T*)&e.v + 4, hi);
    return e;
  } else {
    return Eight<T>{lo, hi};
  }
}
// Two values of byte B of a word of 4-bit codes, in the storage type.
template <typename T, int B> __device__ __forceinline__ uint32_t codes2(uint32_t w, float scale) {
  if constexpr (std::is_same<T, _Float16>::value) return __builtin_bit_cast(uint32_t, (half2v)__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, B));
  else return __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}
template <typename T> __device__ __forceinline__ u32x4 codes8(uint32_t w, float scale) {
  return u32x4{codes2<T, 0>(w, scale), codes2<T, 1>(w, scale), codes2<T, 2>(w, scale), codes2<T, 3>(w, scale)};
}
__device__ __forceinline__ float exp_scale(uint32_t e) { return __uint_as_float(e << 23); }

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const void* base, long long bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)bytes, BUF_FLAGS);
}

// Keys of one tile of 32 as they come from memory, and as the operand of S^T: lane (key % 16, group g).
// Which values of dim a lane holds: 8 from 32 s + 8 g in step s; of 4-bit codes DP / 4 consecutive ones from g DP / 4.
template <typename T, int FORMAT, int DP> struct Keys;
template <typename T, int DP> struct Keys<T, KV_PLAIN, DP> {
  static constexpr int STEPS = DP / 32, ES = sizeof(T), VECS = ES / 2;      // 16-byte vectors per operand
  u32x4 raw[2][STEPS][VECS];
  int off[STEPS];                                          // bytes inside a row; beyond dim: outside every buffer
  __device__ __forceinline__ void init(const AttendArgs& a, int g) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) off[s] = 32 * s + 8 * g < a.dim ? (32 * s + 8 * g) * ES : OOB;
  }
  __device__ __forceinline__ void load(const AttendArgs& a, int head, long long row0, int rows, int col) {
    const __amdgpu_buffer_rsrc_t r = buffer_at(a.k + head * a.k_head + row0 * a.k_row, rows > 0 ? (rows - 1) * a.k_row + a.dim * ES : 0);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int e = 0; e < VECS; ++e) {
          const int o = (16 * h + col) * (int)a.k_row + off[s] + 16 * e;
          raw[h][s][e] = __builtin_amdgcn_raw_buffer_load_b128(r, off[s] == OOB ? OOB : o, 0, 0);
        }
  }
  __device__ __forceinline__ Eight<T> operand(int h, int s) const {
    if constexpr (ES == 2) return Eight<T>{raw[h][s][0]};
    else return Eight<T>{__builtin_bit_cast(floatx4, raw[h][s][0]), __builtin_bit_cast(floatx4, raw[h][s][1])};
  }
  static __device__ __forceinline__ int q_dim(int s, int g) { return 32 * s + 8 * g; }
};
template <typename T, int DP> struct Keys<T, KV_CACHE4, DP> {
  static constexpr int STEPS = DP / 32;
  uint32_t raw[2][STEPS]; uint32_t exp[2];
  int off, eoff;
  __device__ __forceinline__ void init(const AttendArgs& a, int g) {
    const bool in = g * (DP / 4) < a.dim;
    off = in ? g * (DP / 8) : OOB;
    eoff = in ? g * (DP / 4) / 32 : OOB;
  }
  __device__ __forceinline__ void load(const AttendArgs& a, int head, long long row0, int rows, int col) {
    const __amdgpu_buffer_rsrc_t r = buffer_at(a.k + head * a.k_head + row0 * a.k_row, rows > 0 ? (rows - 1) * a.k_row + a.dim / 2 : 0);
    const __amdgpu_buffer_rsrc_t re = buffer_at(a.k_exp + head * a.ke_head + row0 * a.ke_row, rows > 0 ? (rows - 1) * a.ke_row + a.dim / 32 : 0);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int key = 16 * h + col, o = off == OOB ? OOB : key * (int)a.k_row + off;
      if constexpr (DP == 128) {
        const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, 0);
#pragma unroll
        for (int s = 0; s < 4; ++s) raw[h][s] = w[s];
      } else {
        const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(r, o, 0, 0);
        raw[h][0] = w[0]; raw[h][1] = w[1];
      }
      exp[h] = __builtin_amdgcn_raw_buffer_load_b8(re, eoff == OOB ? OOB : key * (int)a.ke_row + eoff, 0, 0);
    }
  }
  __device__ __forceinline__ Eight<T> operand(int h, int s) const { return Eight<T>{codes8<T>(raw[h][s], exp_scale(exp[h]))}; }
  static __device__ __forceinline__ int q_dim(int s, int g) { return g * (DP / 4) + 8 * s; }
};

// Values of the same tile.  A lane (column c, group g) loads the PER = DP / 16 consecutive values from PER c of its eight keys; operand t of
// V^T is then value t of each: row c of the product is element PER c + t of dim.
template <typename T, int FORMAT, int DP> struct Values;
template <typename T, int DP> struct Values<T, KV_PLAIN, DP> {
  static constexpr int PER = DP / 16, ES = sizeof(T), WORDS = PER * ES / 4;
  uint32_t raw[8][WORDS];
  __device__ __forceinline__ void load(const AttendArgs& a, int head, long long row0, int rows, int col, int g) {
    const __amdgpu_buffer_rsrc_t r = buffer_at(a.v + head * a.v_head + row0 * a.v_row, rows > 0 ? (rows - 1) * a.v_row + a.dim * ES : 0);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int o = ((j < 4 ? 0 : 12) + 4 * g + j) * (int)a.v_row + col * PER * ES;
#pragma unroll
      for (int w = 0; w < WORDS; w += 4) {
        if (WORDS - w >= 4) {
          const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(r, o + 4 * w, 0, 0);
#pragma unroll
          for (int e = 0; e < 4; ++e) raw[j][w + e] = x[e];
        } else if (WORDS - w == 3) {
          const u32x3 x = __builtin_amdgcn_raw_buffer_load_b96(r, o + 4 * w, 0, 0);
#pragma unroll
          for (int e = 0; e < 3; ++e) raw[j][w + e] = x[e];
        } else {
          const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(r, o + 4 * w, 0, 0);
          raw[j][w] = x[0]; raw[j][w + 1] = x[1];
        }
      }
    }
  }
  __device__ __forceinline__ void hide(int j, bool keep) {
#pragma unroll
    for (int w = 0; w < WORDS; ++w) raw[j][w] = keep ? raw[j][w] : 0u;
  }
  template <int t> __device__ __forceinline__ Eight<T> operand() const {
    if constexpr (ES == 2) {
      constexpr uint32_t pick = t % 2 ? 0x07060302u : 0x05040100u;          // the two upper or the two lower halves
      Eight<T> e;
#pragma unroll
      for (int i = 0; i < 4; ++i) e.v[i] = __builtin_amdgcn_perm(raw[2 * i + 1][t / 2], raw[2 * i][t / 2], pick);
      return e;
    } else {
      Eight<T> e;
#pragma unroll
      for (int j = 0; j < 4; ++j) { e.lo[j] = __uint_as_float(raw[j][t]); e.hi[j] = __uint_as_float(raw[4 + j][t]); }
      return e;
    }
  }
};
template <typename T, int DP> struct Values<T, KV_CACHE4, DP> {
  static constexpr int PER = DP / 16;
  uint32_t raw[8], exp[8];
  __device__ __forceinline__ void load(const AttendArgs& a, int head, long long row0, int rows, int col, int g) {
    const __amdgpu_buffer_rsrc_t r = buffer_at(a.v + head * a.v_head + row0 * a.v_row, rows > 0 ? (rows - 1) * a.v_row + a.dim / 2 : 0);
    const __amdgpu_buffer_rsrc_t re = buffer_at(a.v_exp + head * a.ve_head + row0 * a.ve_row, rows > 0 ? (rows - 1) * a.ve_row + a.dim / 32 : 0);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int key = (j < 4 ? 0 : 12) + 4 * g + j, o = key * (int)a.v_row + col * PER / 2;
      if constexpr (PER == 8) raw[j] = __builtin_amdgcn_raw_buffer_load_b32(r, o, 0, 0);
      else raw[j] = __builtin_amdgcn_raw_buffer_load_b16(r, o, 0, 0);
      exp[j] = __builtin_amdgcn_raw_buffer_load_b8(re, key * (int)a.ve_row + col * PER / 32, 0, 0);
    }
  }
  __device__ __forceinline__ void hide(int j, bool keep) { raw[j] = keep ? raw[j] : 0u; exp[j] = keep ? exp[j] : 0u; }
  template <int t> __device__ __forceinline__ Eight<T> operand() const {
    constexpr uint32_t pick = t % 2 ? 0x07060302u : 0x05040100u;
    Eight<T> e;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      e.v[i] = __builtin_amdgcn_perm(codes2<T, t / 2>(raw[2 * i + 1], exp_scale(exp[2 * i + 1])), codes2<T, t / 2>(raw[2 * i], exp_scale(exp[2 * i])), pick);
    return e;
  }
};

template <typename T, int FORMAT, int DP, int RT, int t> __device__ __forceinline__ void add_values(const Values<T, FORMAT, DP>& v, const Eight<T>* p, floatx4 (*acc)[DP / 16]) {
  if constexpr (t < DP / 16) {
    const Eight<T> a = v.template operand<t>();
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[r][t] = mma<T>(a, p[r], acc[r][t]);
    add_values<T, FORMAT, DP, RT, t + 1>(v, p, acc);
  }
}

// Scaled weights of a row's part of the keys become one result: out and lse, or a part for attend_join_kernel.
template <typename T, int PER>
__device__ __forceinline__ void finish_row(const AttendArgs& a, int part, bool whole, long long q_row, int head, int d0, bool first, const float* o, float ref, float sum) {
  if (!whole) {
    const long long at = ((long long)part * a.n_q + q_row) * a.q_heads + head;
    if (first) a.part_ml[at] = make_float2(ref, sum);
    float* y = a.part_o + at * a.dim + d0;
#pragma unroll
    for (int e = 0; e < PER; e += 2)
      if (d0 + e < a.dim) *(float2*)(y + e) = make_float2(o[e], o[e + 1]);
    return;
  }
  const float r = sum != 0.f ? 1.0f / sum : 0.f;         // a sum that is NaN stays one
  if (first && a.lse) a.lse[q_row * a.q_heads + head] = sum != 0.f ? (ref + log2f(sum)) * 0.693147180559945f : -INFINITY;
  T* y = (T*)a.out + q_row * a.out_row + head * a.out_head + d0;
  typedef T t2 __attribute__((ext_vector_type(2)));
  if constexpr (PER % 4 == 0) {
#pragma unroll
    for (int e = 0; e < PER; e += 4)
      if (d0 + e < a.dim) store4<T>(y + e, floatx4{o[e] * r, o[e + 1] * r, o[e + 2] * r, o[e + 3] * r});
  } else {
#pragma unroll
    for (int e = 0; e < PER; e += 2)
      if (d0 + e < a.dim) *(t2*)(y + e) = t2{(T)(o[e] * r), (T)(o[e + 1] * r)};
  }
}

// A wavefront has RT times 16 rows and walks over tiles of 32 keys, which it loads from memory to registers in the order of the operands: no
// LDS and no barrier on the way, the next tile's loads are in flight while one is computed.  SHARE: the four wavefronts of
// a block have the same rows and every fourth tile each, and add up in LDS at the end (few rows: what bounds it is reading the keys, and
// more wavefronts have more loads in flight); otherwise each has rows of its own.  RT = 2: two blocks of rows use each operand that has been loaded, and
// converted or put in order.
template <typename T, int FORMAT, int DP, bool SHARE, bool MASK, int RT>
__global__ __launch_bounds__(256, RT == 2 && sizeof(T) == 4 && DP == 128 ? 1 : 2) void attend_direct_kernel(AttendArgs a) {
  constexpr int STEPS = DP / 32, PER = DP / 16, WAVES = SHARE ? 4 : 1;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
  // what a block (SHARE) or a wavefront does: some rows of a sequence and key head
  const Piece pc = piece_of(a, SHARE ? blockIdx.x : blockIdx.x * 4 + wave, SHARE && a.by_die);
  const int b = pc.seq, kv_head = pc.head, part = pc.part, row0 = pc.block * 16 * RT;
  Span sp;
  if (b >= a.n_seq || !span_of(a, b, &sp)) return;
  const int rows = sp.n_q * a.group;
  if (row0 >= rows || part >= parts_of(sp.n_kv, a.part_keys)) return;      // SHARE: the whole block
  const bool whole = sp.n_kv <= a.part_keys;

  const int tiles = (sp.n_kv + 31) / 32, per_part = a.part_keys / 32;
  const int first = part * per_part, last = min(tiles, first + per_part);      // first .. last - 1

  Keys<T, FORMAT, DP> keys;
  Values<T, FORMAT, DP> vals;
  Eight<T> q[RT][STEPS];
  keys.init(a, g);
  uint32_t mask_byte = 0;
  auto keys_left = [&](int t) { return t < last ? min(32, sp.n_kv - 32 * t) : 0; };
  auto load_mask = [&](int t) {
    if constexpr (MASK) mask_byte = __builtin_amdgcn_raw_buffer_load_b8(buffer_at(a.mask + sp.kv0 + 32ll * t, keys_left(t)), lane, 0, 0);
  };
  int t = first + (SHARE ? wave : 0);
  keys.load(a, kv_head, sp.kv0 + 32ll * t, keys_left(t), col);
  vals.load(a, kv_head, sp.kv0 + 32ll * t, keys_left(t), col, g);
  load_mask(t);
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = row0 + 16 * r + col, qi = (int)fast_div((unsigned)row, a.div_group), head = kv_head * a.group + row - qi * a.group;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int d = Keys<T, FORMAT, DP>::q_dim(s, g);
      const T* p = (const T*)a.q + (sp.q0 + (long long)qi) * a.q_row + head * a.q_head + d;
      const bool in = row < rows && d < a.dim;
      if constexpr (sizeof(T) == 2) q[r][s].v = in ? *(const u32x4*)p : u32x4{0, 0, 0, 0};
      else { q[r][s].lo = in ? *(const floatx4*)p : floatx4{0, 0, 0, 0}; q[r][s].hi = in ? *(const floatx4*)(p + 4) : floatx4{0, 0, 0, 0}; }
    }
  }

  floatx4 acc[RT][PER];
  float ref[RT], sum[RT];                  // the reference in units of the raw score: weights are exp2((s - ref) scale2)
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    ref[r] = -INFINITY; sum[r] = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[r][i] = floatx4{0, 0, 0, 0};
  }
  const float c = a.scale2;

  for (; t < last; t += WAVES) {
    const int n = keys_left(t);
    const unsigned seen = MASK ? (unsigned)__ballot(mask_byte != 0) : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1;
    floatx4 st[RT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int r = 0; r < RT; ++r) st[r][h] = floatx4{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        const Eight<T> k = keys.operand(h, s);
#pragma unroll
        for (int r = 0; r < RT; ++r) st[r][h] = mma<T>(k, q[r][s], st[r][h]);
      }
    }
    keys.load(a, kv_head, sp.kv0 + 32ll * (t + WAVES), keys_left(t + WAVES), col);
    load_mask(t + WAVES);
    if (seen != 0xFFFFFFFFu) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool keep = seen >> (16 * h + 4 * g + i) & 1;
#pragma unroll
          for (int r = 0; r < RT; ++r) st[r][h][i] = keep ? st[r][h][i] : -INFINITY;
          if (MASK) vals.hide(4 * h + i, keep);               // beyond the last key zeros were read
        }
    }
    // The reference follows the largest score only where that is more than 2^8 above it: weights up to 2^8 cost no precision,
    // and the sums seldom have to be scaled.
    float top[RT];
    bool over = false;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      top[r] = fmaxf(fmaxf(fmaxf(st[r][0][0], st[r][0][1]), fmaxf(st[r][0][2], st[r][0][3])), fmaxf(fmaxf(st[r][1][0], st[r][1][1]), fmaxf(st[r][1][2], st[r][1][3])));
      over = over || (top[r] - ref[r]) * c > 8.0f;
    }
    if (__any(over)) {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        float m = fmaxf(top[r], __shfl_xor(top[r], 16));
        m = fmaxf(ref[r], fmaxf(m, __shfl_xor(m, 32)));
        const float alpha = m == ref[r] ? 1.0f : __builtin_amdgcn_exp2f((ref[r] - m) * c);
        ref[r] = m;
        sum[r] *= alpha;
#pragma unroll
        for (int i = 0; i < PER; ++i) acc[r][i] *= alpha;
      }
    }
    Eight<T> p[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const float refc = ref[r] == -INFINITY ? 0.f : ref[r] * c;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) { st[r][h][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[r][h][i], c, -refc)); sum[r] += st[r][h][i]; }
      // The second product takes operands of T, so the weights are rounded to it (their sum is not).  Outputs, which are rounded to T themselves, are then
      // off by 2.3e-3 of their size in bf16 instead of 1.7e-3, 2.4e-4 instead of 2.1e-4 in fp16; with the weights' remainders it would be one and a half times the matrix instructions.
      p[r] = eight_of<T>(st[r][0], st[r][1]);
    }
    add_values<T, FORMAT, DP, RT, 0>(vals, p, acc);
    vals.load(a, kv_head, sp.kv0 + 32ll * (t + WAVES), keys_left(t + WAVES), col, g);
  }

  constexpr int LD = DP + 4;
  __shared__ float so[SHARE ? 4 : 1][SHARE ? 16 : 1][LD];
  __shared__ float2 sm[SHARE ? 4 : 1][SHARE ? 16 : 1];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    sum[r] += __shfl_xor(sum[r], 16);
    sum[r] += __shfl_xor(sum[r], 32);
    const float refc = ref[r] == -INFINITY ? -INFINITY : ref[r] * c;
    // element of dim of acc[r][t][i]: PER (4 g + i) + t
    if constexpr (!SHARE) {
      const int row = row0 + 16 * r + col, qi = (int)fast_div((unsigned)row, a.div_group);
      if (row >= rows) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float o[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] = acc[r][e][i];
        finish_row<T, PER>(a, part, whole, sp.q0 + (long long)qi, kv_head * a.group + row - qi * a.group, PER * (4 * g + i), g == 0 && i == 0, o, refc, sum[r]);
      }
    } else {
      if (row0 + 16 * r >= rows) break;                    // the same for the whole block
      if (r) __syncthreads();                              // the rows before have been read
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < PER; e += 2) *(float2*)&so[wave][col][PER * (4 * g + i) + e] = make_float2(acc[r][e][i], acc[r][e + 1][i]);
      if (g == 0) sm[wave][col] = make_float2(refc, sum[r]);
      __syncthreads();
      const int x = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * PER, row = row0 + 16 * r + x;
      if (row >= rows) continue;
      float m = -INFINITY, total = 0.f, o[PER];
#pragma unroll
      for (int w = 0; w < 4; ++w) m = fmaxf(m, sm[w][x].x);
#pragma unroll
      for (int e = 0; e < PER; ++e) o[e] = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float2 y = sm[w][x];
        const float f = y.x == m ? 1.0f : __builtin_amdgcn_exp2f(y.x - m);
        total += y.y * f;
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] += so[w][x][d0 + e] * f;
      }
      const int qi = (int)fast_div((unsigned)row, a.div_group);
      finish_row<T, PER>(a, part, whole, sp.q0 + (long long)qi, kv_head * a.group + row - qi * a.group, d0, d0 == 0, o, m, total);
    }
  }
}

template <typename T, int FORMAT, int DP, bool MASK>
hipError_t launch_direct_masked(int how, const AttendArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.blocks);
  if (how == DIRECT_OWN) hipLaunchKernelGGL((attend_direct_kernel<T, FORMAT, DP, false, MASK, 1>), grid, dim3(256), 0, s, a);
  else if (how == DIRECT_SHARE) hipLaunchKernelGGL((attend_direct_kernel<T, FORMAT, DP, true, MASK, 1>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((attend_direct_kernel<T, FORMAT, DP, true, MASK, 2>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename T, int FORMAT, int DP>
hipError_t launch_direct(int how, const AttendArgs& a, hipStream_t s) {
  return a.mask ? launch_direct_masked<T, FORMAT, DP, true>(how, a, s) : launch_direct_masked<T, FORMAT, DP, false>(how, a, s);
}
template <typename T>
hipError_t launch_attend_direct(int format, int how, const AttendArgs& a, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (format == KV_CACHE4) return a.dim <= 64 ? launch_direct<T, KV_CACHE4, 64>(how, a, s) : launch_direct<T, KV_CACHE4, 128>(how, a, s);
  }
  if (a.dim <= 64) return launch_direct<T, KV_PLAIN, 64>(how, a, s);
  if (a.dim <= 96) return launch_direct<T, KV_PLAIN, 96>(how, a, s);
  return launch_direct<T, KV_PLAIN, 128>(how, a, s);
}
#endif

}  // namespace octo
