// octo_op_attend for many rows: a block of four wavefronts shares tiles of 64 keys and values in LDS.
//
// What bounds it is the arithmetic: 4 x rows x keys x dim operations on the matrix cores and, beside them, one exponential per row
// and key, which the vector units take longer for than the matrix cores for the products of 64 dims.  A wavefront has 32 rows, S^T = K Q^T
// and O^T = V^T P^T in blocks of 32 x 32 x 16, so that a lane has half the scores of one row, the reference and the sum are its own (one
// exchange with lane ^ 32 where the reference moves), and the weights go into the second product from the registers they are made in: slot j of
// lane half h and step k stands for key 16 k + 4 h + j (j < 4) or 16 k + 8 + 4 h + j - 4.  Two wavefronts per SIMD: one's exponentials run beside the other's
// products.
//
// LDS.  Two stages; loads of the next tile go straight to LDS while one is computed (keys of 4 bits through registers, where they become 16 bits).  Rows
// of 16-byte chunks, chunk c of row r at c ^ swizzle(r): for keys the low bits of r, so that eight rows' equal chunks lie in different
// banks; for values, read transposed four rows by 16 columns at a time, bits that put the four rows into different banks.
#pragma once
#include "attend.h"

namespace octo {

hipError_t launch_attend_tile_f16(int format, const AttendArgs& a, hipStream_t s);
hipError_t launch_attend_tile_bf16(int format, const AttendArgs& a, hipStream_t s);

#ifdef __HIPCC__
typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) unsigned char LdsByte;

template <int RB> __device__ __forceinline__ int swizzle_k(int row) { return row & (RB / 16 - 1); }
template <int RB> __device__ __forceinline__ int swizzle_v(int row) { return RB == 256 ? (row & 3) << 2 : (row & 2) << 1; }

// Which piece of work a block has, where the lengths on the device decide: every block looks at all sequences (up to 256, one a thread), takes for the
// longest part of a sequence the number of tiles with the least estimated end - one, two or three rounds of blocks on all units, or no
// parts at all -, and finds its sequence by a running sum.  With parts of a fixed number of keys ragged sequences leave a last round half empty:
// 60 drawn calls of more than 1000 keys take 4 to 5 % less in the mean, ragged ones up to a third (9 questions of up to 79 tokens over up to 22497 keys of 4 bits 193 -> 134 us, 29 texts of
// up to 1053 tokens over up to 7029 keys 420 -> 336), single ones more (136 x 258 over up to 10341 321 -> 375).
// Where the sequences turn out to be of equal length, the host's number of parts stands (even_tiles).
struct CutPiece { int seq, head, block, part, part_keys, q0, n_q, n_kv; long long kv0; };
__device__ __forceinline__ bool cut_piece(const AttendArgs& a, CutPiece* piece, float (*red)[8], int* ends) {
  const int i = threadIdx.x, lane = i & 63, wave = i >> 6;
  Span sp;
  const bool has = i < a.n_seq && span_of(a, i, &sp);
  const int blocks = has ? (sp.n_q * a.group + 127) / 128 : 0, tiles = has ? (sp.n_kv + 63) / 64 : 0;
  if (i == 0) piece->seq = -1;
  float work = (float)blocks * tiles, whole = (float)blocks;
  int longest = tiles;
  for (int d = 1; d < 64; d *= 2) { work += __shfl_xor(work, d); whole += __shfl_xor(whole, d); longest = max(longest, __shfl_xor(longest, d)); }
  if (lane == 0) { red[wave][0] = work; red[wave][1] = whole; ends[wave] = longest; }
  __syncthreads();
  work = (red[0][0] + red[1][0] + red[2][0] + red[3][0]) * a.kv_heads;
  whole = (red[0][1] + red[1][1] + red[2][1] + red[3][1]) * a.kv_heads;
  longest = max(max(ends[0], ends[1]), max(ends[2], ends[3]));      // ends: free again after the next barrier
  const CutSums sums{work, whole, longest};
  const float slots = (float)a.slots;
  const int least = cut_least(sums, a.n_split);
  int most[3];
  float pieces[3];
#pragma unroll
  for (int c = 0; c < 3; ++c) {
    most[c] = cut_most(sums, slots, least, c);
    pieces[c] = (float)(blocks * (tiles > most[c] ? (tiles + most[c] - 1) / most[c] : 1));
    for (int d = 1; d < 64; d *= 2) pieces[c] += __shfl_xor(pieces[c], d);
    if (lane == 0) red[wave][3 + c] = pieces[c];
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < 3; ++c) pieces[c] = (red[0][3 + c] + red[1][3 + c] + red[2][3 + c] + red[3][3 + c]) * a.kv_heads;
  const int part = cut_tiles(sums, most, pieces, slots, least, a.even_tiles, (float)a.n_seq * a.row_blocks * a.kv_heads, (float)a.blocks);
  if (blockIdx.x == 0 && i == 0) *a.cut_tiles = part;
  // whose piece is it
  const int part_keys = even_part(has ? sp.n_kv : 0, part), mine = has ? blocks * a.kv_heads * parts_of(sp.n_kv, part_keys) : 0;
  int end = mine;
  for (int d = 1; d < 64; d *= 2) { const int o = __shfl_up(end, d); if (lane >= d) end += o; }
  if (lane == 63) ends[wave] = end;
  __syncthreads();
  for (int w = 0; w < wave; ++w) end += ends[w];
  const int at = (int)blockIdx.x - (end - mine);
  if (at >= 0 && at < mine) {
    // sets of keys (head, part) eight at a time: the blocks of rows of a set are eight numbers apart, on one die
    const int sets = mine / blocks, full = sets / 8 * 8 * blocks, o = at - full;
    const int set = at < full ? at / (8 * blocks) * 8 + at % 8 : sets / 8 * 8 + o % (sets % 8 ? sets % 8 : 1);
    const int block = at < full ? at % (8 * blocks) / 8 : o / (sets % 8 ? sets % 8 : 1);
    *piece = CutPiece{i, set % a.kv_heads, block, set / a.kv_heads, part_keys, sp.q0, sp.n_q, sp.n_kv, sp.kv0};
  }
  __syncthreads();
  return piece->seq >= 0;
}

// MASK: some keys are hidden by a mask; without one only the end of the last tile is, and what is read beyond it is zero.
template <typename T, int FORMAT, int DP, bool MASK>
__global__ __launch_bounds__(256, 2) void attend_tile_kernel(AttendArgs a) {
  constexpr int TK = 64, RB = DP <= 64 ? 128 : 256, CH = RB / 16, STEPS = DP / 16, DT = DP / 32, TILE = TK * RB;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILE];          // keys, keys, values, values
  __shared__ CutPiece cut;
  __shared__ float cut_red[4][8];
  __shared__ int cut_ends[4];
  int b, kv_head, part, block, part_keys = a.part_keys;
  Span sp;
  if (a.cut) {
    if (!cut_piece(a, &cut, cut_red, cut_ends)) return;
    b = __builtin_amdgcn_readfirstlane(cut.seq); kv_head = __builtin_amdgcn_readfirstlane(cut.head); part = __builtin_amdgcn_readfirstlane(cut.part);
    block = __builtin_amdgcn_readfirstlane(cut.block); part_keys = __builtin_amdgcn_readfirstlane(cut.part_keys);
    sp.q0 = __builtin_amdgcn_readfirstlane(cut.q0); sp.n_q = __builtin_amdgcn_readfirstlane(cut.n_q); sp.n_kv = __builtin_amdgcn_readfirstlane(cut.n_kv);
    sp.kv0 = (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(cut.kv0 >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)cut.kv0));
  } else {
    const Piece pc = piece_of(a, blockIdx.x, a.by_die);
    b = pc.seq; kv_head = pc.head; part = pc.part; block = pc.block;
    if (b >= a.n_seq || !span_of(a, b, &sp)) return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, half = lane >> 5;
  const int rows = sp.n_q * a.group;
  if (block * 128 >= rows || part >= parts_of(sp.n_kv, part_keys)) return;
  const bool whole = sp.n_kv <= part_keys;
  const int row = block * 128 + wave * 32 + l32;
  const bool has_row = row < rows, busy = block * 128 + wave * 32 < rows;      // a wavefront without rows loads and waits with the others
  const int qi = (int)fast_div((unsigned)row, a.div_group), head = kv_head * a.group + row - qi * a.group;
  const long long q_row = sp.q0 + qi;

  const int tiles = (sp.n_kv + TK - 1) / TK, per_part = part_keys / TK;
  const int first = part * per_part, last = min(tiles, first + per_part);
  auto keys_left = [&](int t) { return t < last ? min(TK, sp.n_kv - TK * t) : 0; };
  uint32_t mask_byte = 0;
  auto load_mask = [&](int t) {
    if constexpr (MASK) mask_byte = __builtin_amdgcn_raw_buffer_load_b8(buffer_at(a.mask + sp.kv0 + (long long)TK * t, keys_left(t)), lane, 0, 0);
  };
  auto seen_of = [&](int t) -> unsigned long long {
    if constexpr (MASK) return __ballot(mask_byte != 0);
    const int n = keys_left(t);
    return n >= TK ? ~0ull : (1ull << n) - 1;
  };

  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(LdsByte*)smem);
  const char* const k_base = a.k + kv_head * a.k_head;
  const char* const v_base = a.v + kv_head * a.v_head;

  // plain: what a lane loads, NI instructions of 64 chunks a wavefront and tensor
  constexpr int NI = TILE / 4096;
  // 4 bits: a thread takes 32 values of a key
  constexpr int PARTS = DP / 32;
  u32x4 held[2]; uint32_t held_exp[2];

  // K of tile t, V of tile t: to a stage of LDS (plain), or to registers, from which place_tile takes them there
  auto load_tile = [&](int t, int stage, bool is_v, unsigned long long seen) __attribute__((always_inline)) {
    const int n = keys_left(t);
    const long long row0 = sp.kv0 + (long long)TK * t, pitch = is_v ? a.v_row : a.k_row;
    const __amdgpu_buffer_rsrc_t rc = buffer_at((is_v ? v_base : k_base) + row0 * pitch, n > 0 ? (n - 1) * pitch + (FORMAT == KV_CACHE4 ? a.dim / 2 : a.dim * 2) : 0);
    if constexpr (FORMAT == KV_PLAIN) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int r = (wave * NI + i) * (64 / CH) + lane / CH, ch = (lane % CH) ^ (is_v ? swizzle_v<RB>(r) : swizzle_k<RB>(r));
        const bool see = !MASK || !is_v || (seen >> r & 1);         // what a hidden key holds is replaced in the scores
        const int o = see && ch * 8 < a.dim ? r * (int)pitch + ch * 16 : OOB;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :: "s"(lds + (is_v ? 2 * TILE : 0) + stage * TILE + (wave * NI + i) * 1024), "v"(o), "s"(rc) : "memory");
      }
    } else {
      const long long epitch = is_v ? a.ve_row : a.ke_row;
      const __amdgpu_buffer_rsrc_t re = buffer_at((is_v ? a.v_exp + kv_head * a.ve_head : a.k_exp + kv_head * a.ke_head) + row0 * epitch, n > 0 ? (n - 1) * epitch + a.dim / 32 : 0);
      const int r = (int)threadIdx.x / PARTS % TK, p = (int)threadIdx.x % PARTS;
      const bool see = (!MASK || !is_v || (seen >> r & 1)) && p * 32 < a.dim && (int)threadIdx.x < TK * PARTS;
      held[is_v] = __builtin_amdgcn_raw_buffer_load_b128(rc, see ? r * (int)pitch + p * 16 : OOB, 0, 0);
      held_exp[is_v] = __builtin_amdgcn_raw_buffer_load_b8(re, see ? r * (int)epitch + p : OOB, 0, 0);
    }
  };
  auto place_tile = [&](int stage, bool is_v) __attribute__((always_inline)) {
    if constexpr (FORMAT == KV_CACHE4) {
      const int r = (int)threadIdx.x / PARTS % TK, p = (int)threadIdx.x % PARTS;
      if ((int)threadIdx.x < TK * PARTS) {
        unsigned char* const to = smem + (is_v ? 2 * TILE : 0) + stage * TILE + r * RB;
        const int sw = is_v ? swizzle_v<RB>(r) : swizzle_k<RB>(r);
        const float scale = exp_scale(held_exp[is_v]);
#pragma unroll
        for (int e = 0; e < 4; ++e) *(u32x4*)(to + ((4 * p + e) ^ sw) * 16) = codes8<T>(held[is_v][e], scale);
      }
    }
  };

  load_mask(first);
  load_tile(first, 0, false, 0);
  u32x4 q[STEPS];
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int d = 16 * s + 8 * half;
    q[s] = has_row && d < a.dim ? *(const u32x4*)((const T*)a.q + q_row * a.q_row + head * a.q_head + d) : u32x4{0, 0, 0, 0};
  }
  unsigned long long seen = seen_of(first), seen_next;
  load_tile(first, 0, true, seen);
  load_mask(first + 1);
  place_tile(0, false);
  load_tile(first + 1, 1, false, 0);
  place_tile(0, true);
  place_tile(1, false);

  // addresses of a lane's operands inside a stage: of the first step; the others differ in the bits of the chunk
  const int at_k = l32 * RB + (half ^ swizzle_k<RB>(l32)) * 16;
  const int vi = lane & 15, vr = 4 * half + vi / 4;                // key vr (+ 16 k, + 8), columns 16 (lane / 16 % 2) + 4 (vi % 4) ..
  const int at_v = vr * RB + (((lane >> 4 & 1) * 2 + (vi >> 1 & 1)) ^ swizzle_v<RB>(vr)) * 16 + (vi & 1) * 8;

  floatx16 acc[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
  float ref = -INFINITY, sum = 0.f;
  const float c = a.scale2;

  floatx16 st[2];
  auto scores = [&](const unsigned char* ks, floatx16* to) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 16; ++i) to[h][i] = 0.f;
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
      for (int h = 0; h < 2; ++h) to[h] = Elem<T>::mfma(*(const u32x4*)(ks + (at_k ^ 32 * s) + h * 32 * RB), q[s], to[h]);
  };
  // One tile: the exponentials of its scores beside the products of the next tile's, then its values.
  auto step = [&](int t, auto more) __attribute__((always_inline)) {
    const int stage = (t - first) & 1;
    // the next keys and these values have landed for all wavefronts, and all are done with the stages that are loaded next
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    seen_next = seen_of(t + 1);
    if constexpr (more()) {
      load_tile(t + 2, stage, false, 0);
      load_tile(t + 1, stage ^ 1, true, seen_next);
      load_mask(t + 2);
    }
    const unsigned char* const vs = smem + 2 * TILE + stage * TILE;
    if (busy) {
    if (seen != ~0ull) {
      // score i of half h belongs to key 32 h + 8 (i / 4) + i % 4 in lanes 0 .. 31 and to the key four further on in the others: which lanes keep it is made of
      // two bits by the scalar unit (three vector instructions a score otherwise)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int bit = 8 * (i / 4) + i % 4, bits = (int)(h ? seen >> 32 : seen);
          const unsigned long long keep = (unsigned)((bits << (31 - bit)) >> 31) | (unsigned long long)(unsigned)((bits << (27 - bit)) >> 31) << 32;
          st[h][i] = __builtin_amdgcn_inverse_ballot_w64(keep) ? st[h][i] : -INFINITY;
        }
    }
    float top = st[0][0];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, st[h][i]);
    if (__any((top - ref) * c > 8.0f)) {                           // as in attend_direct_kernel
      const float m = fmaxf(ref, fmaxf(top, __shfl_xor(top, 32)));
      const float alpha = m == ref ? 1.0f : __builtin_amdgcn_exp2f((ref - m) * c);
      ref = m;
      sum *= alpha;
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[d] *= alpha;
    }
    // From here to the end of the products the wavefront goes before the other of its SIMD, which is then at its loads and comparisons or waits
    // (2 x 2048 queries over 12800 keys 777 -> 762 us, 732 together with the line drawn between exponentials and values below).
    __builtin_amdgcn_s_setprio(1);
    const float refc = ref == -INFINITY ? 0.f : ref * c;
    floatx16 nx[2];
    if constexpr (more()) scores(smem + (stage ^ 1) * TILE, nx);
    float add[2] = {0.f, 0.f};
    u32x4 p[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) { w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[k / 2][8 * (k % 2) + i], c, -refc)); add[i & 1] += w[i]; }
      // rounded to T, as in attend_direct_kernel
      store4<T>((T*)&p[k], floatx4{w[0], w[1], w[2], w[3]});
      store4<T>((T*)&p[k] + 4, floatx4{w[4], w[5], w[6], w[7]});
    }
    sum += add[0] + add[1];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const short4v v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(vs + (at_v ^ 64 * d) + 16 * k * RB));
        const short4v v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(vs + (at_v ^ 64 * d) + (16 * k + 8) * RB));
        const u32x2 w0 = __builtin_bit_cast(u32x2, v0), w1 = __builtin_bit_cast(u32x2, v1);
        acc[d] = Elem<T>::mfma(u32x4{w0[0], w0[1], w1[0], w1[1]}, p[k], acc[d]);
      }
    if constexpr (more()) { st[0] = nx[0]; st[1] = nx[1]; }
    __builtin_amdgcn_s_setprio(0);
    }
    if constexpr (more()) {
      place_tile(stage, false);
      place_tile(stage ^ 1, true);
    }
    seen = seen_next;
  };
  if (first < last) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    scores(smem, st);
    for (int t = first; t < last - 1; ++t) step(t, std::true_type{});
    step(last - 1, std::false_type{});
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                 // loads issued past the last tile write zeros into LDS
  if (!has_row) return;
  sum += __shfl_xor(sum, 32);                                      // both lanes of a row are here
  const float refc = ref == -INFINITY ? -INFINITY : ref * c;

  // element of dim of acc[d][i]: 32 d + 8 (i / 4) + 4 half + i % 4
  if (!whole) {
    const long long at = ((long long)part * a.n_q + q_row) * a.q_heads + head;
    if (!half) a.part_ml[at] = make_float2(refc, sum);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int e = 32 * d + 2 * i + 4 * half;
        if (e < a.dim) *(floatx4*)(a.part_o + at * a.dim + e) = floatx4{acc[d][i], acc[d][i + 1], acc[d][i + 2], acc[d][i + 3]};
      }
    return;
  }
  const float r = sum != 0.f ? 1.0f / sum : 0.f;
  if (!half && a.lse) a.lse[q_row * a.q_heads + head] = sum != 0.f ? (refc + log2f(sum)) * 0.693147180559945f : -INFINITY;
  T* const y = (T*)a.out + q_row * a.out_row + head * a.out_head;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 8) {
      // chunks i / 4 and i / 4 + 1 of eight values, half of each here, half in lane ^ 32: afterwards one whole chunk in each
      u32x2 x, z;
      store4<T>((T*)&x, floatx4{acc[d][i] * r, acc[d][i + 1] * r, acc[d][i + 2] * r, acc[d][i + 3] * r});
      store4<T>((T*)&z, floatx4{acc[d][i + 4] * r, acc[d][i + 5] * r, acc[d][i + 6] * r, acc[d][i + 7] * r});
      const auto s0 = __builtin_amdgcn_permlane32_swap(x[0], z[0], false, false), s1 = __builtin_amdgcn_permlane32_swap(x[1], z[1], false, false);
      const int e = 32 * d + 2 * i + 8 * half;
      if (e < a.dim) *(u32x4*)(y + e) = u32x4{s0[0], s1[0], s0[1], s1[1]};
    }
}

template <typename T, int FORMAT, int DP>
hipError_t launch_tile(const AttendArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.blocks);
  if (a.mask) hipLaunchKernelGGL((attend_tile_kernel<T, FORMAT, DP, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((attend_tile_kernel<T, FORMAT, DP, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_attend_tile(int format, const AttendArgs& a, hipStream_t s) {
  if (format == KV_CACHE4) return a.dim <= 64 ? launch_tile<T, KV_CACHE4, 64>(a, s) : a.dim <= 96 ? launch_tile<T, KV_CACHE4, 96>(a, s) : launch_tile<T, KV_CACHE4, 128>(a, s);
  if (a.dim <= 64) return launch_tile<T, KV_PLAIN, 64>(a, s);
  if (a.dim <= 96) return launch_tile<T, KV_PLAIN, 96>(a, s);
  return launch_tile<T, KV_PLAIN, 128>(a, s);
}
#endif

}  // namespace octo
